// RMS norm of every query and key head and the rotary embedding, in one pass:
//   y = x / sqrt(mean(x^2) + eps) * g           (over the head's dh dims)
//   out[i]        = y[i] cos - y[i + dh/2] sin
//   out[i + dh/2] = y[i + dh/2] cos + y[i] sin   (the angle of the token's position)
// Bound by memory: each head row is read once and written once.  DH / 8 lanes
// hold a row, 8 dims each, and a dim's partner lies in the lane that a DPP
// mirror of the row reaches: lane j of the first half holds dims 8 j .., lane
// DH / 8 - 1 - j dims DH / 2 + 8 j ...  So loads and stores are 16 bytes a lane
// over whole cache lines, and neither the rotation nor the sum of squares
// (fp32) leaves the registers.  2048 tokens of 32 + 32 heads, dh = 128, bf16
// (68 MB): 14.8 us, 4.6 TB/s, where three such calls' rows stay in the 256 MB cache,
// nine tenths of what adding two tensors of that size reaches; 19.7 us from and to
// memory; a decode step of four tokens 2.3 us, a launch's own time.
#include "kernels.h"

namespace vla {
namespace {

template <bool F32>
__device__ __forceinline__ void load8(const void* p, int64_t at, float (&x)[8]) {
  if constexpr (F32) {
    const f32x4 a = *(const f32x4*)((const float*)p + at), b = *(const f32x4*)((const float*)p + at + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = a[e], x[4 + e] = b[e];
  } else {
    const u32x4 w = *(const u32x4*)((const bf16_t*)p + at);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[2 * e] = __uint_as_float(w[e] << 16);
      x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
    }
  }
}

// One token per workgroup; its 2048 / DH rows of lanes take the query and key
// heads, two at a time with their loads on their way at once.
template <int DH, bool F32>
__global__ __launch_bounds__(256) void qk_norm_rope_kernel(QkNormArgs a) {
  constexpr int LN = DH / 8, ROWS = 256 / LN, U = 2;
  const int tid = threadIdx.x, j = tid % LN, slot = tid / LN;
  const bool first = j < LN / 2;
  const int i0 = first ? 8 * j : 8 * (LN - 1 - j), d0 = first ? i0 : DH / 2 + i0;
  const int b = div_by(blockIdx.x, a.by_L), t = blockIdx.x - b * a.L, heads = a.H + a.Hkv;
  float x[U][8];
  auto load = [&](int h0) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int h = min(h0 + u * ROWS, heads - 1);  // past the last head: that one again, not stored
      const Heads& in = h < a.H ? a.q : a.k;
      load8<F32>(in.p, b * in.seq + t * in.token + (h < a.H ? h : h - a.H) * in.head + d0, x[u]);
    }
  };
  load(slot);  // beside the position, which the table's loads wait for
  const int pos = a.cos && a.pos ? a.pos[blockIdx.x] : t;
  float c[8], s[8];
  if (a.cos) {
    if (pos < 0 || pos >= a.n_pos) return;
    load8<true>(a.cos, (int64_t)pos * (DH / 2) + i0, c);
    load8<true>(a.sin, (int64_t)pos * (DH / 2) + i0, s);
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] = first ? -s[e] : s[e];
  }
  for (int h0 = slot; h0 < heads; h0 += ROWS * U) {
    if (h0 != slot) load(h0);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int h = h0 + u * ROWS;
      if (h >= heads) break;
      const float* gain = h < a.H ? a.gq : a.gk;
      if (gain) {
        float g[8], sum = 0.f;
        load8<true>(gain, d0, g);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += x[u][e] * x[u][e];
        const float r = 1.f / sqrtf(row_sum<LN>(sum) / DH + a.eps);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[u][e] = x[u][e] * r * g[e];
      }
      if (a.cos) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float partner = dpp<LN == 16 ? 0x140 : 0x141>(x[u][e]);
          x[u][e] = x[u][e] * c[e] + partner * s[e];
        }
      }
      const Heads& out = h < a.H ? a.q_out : a.k_out;
      bf16_t* o = (bf16_t*)out.p + b * out.seq + t * out.token + (h < a.H ? h : h - a.H) * out.head + d0;
      *(u32x4*)o = u32x4{pack_bf2(x[u][0], x[u][1]), pack_bf2(x[u][2], x[u][3]), pack_bf2(x[u][4], x[u][5]),
                         pack_bf2(x[u][6], x[u][7])};
    }
  }
}

template <int DH>
hipError_t launch(const QkNormArgs& a, bool f32, hipStream_t s) {
  const dim3 grid(a.B * a.L), block(256);
  if (f32)
    hipLaunchKernelGGL((qk_norm_rope_kernel<DH, true>), grid, block, 0, s, a);
  else
    hipLaunchKernelGGL((qk_norm_rope_kernel<DH, false>), grid, block, 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t qk_norm_rope(QkNormArgs a, bool f32, int dh, hipStream_t s) {
  a.by_L = fast_div(a.L);
  return dh == 128 ? launch<128>(a, f32, s) : launch<64>(a, f32, s);
}

}  // namespace vla
