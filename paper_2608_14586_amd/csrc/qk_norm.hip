// RMS norm of every query and key head and the rotary embedding, in one pass:
//   y = x / sqrt(mean(x^2) + eps) * g           (over the head's dh dims)
//   out[i]        = y[i] cos - y[i + dh/2] sin
//   out[i + dh/2] = y[i + dh/2] cos + y[i] sin   (the angle of the token's position)
// Bound by memory: each head row is read once and written once.  dh / 8 lanes
// hold a row, each four dims of the first half and their four partners of the
// second, so the rotation stays inside the lane and the loads of the lanes
// side by side still cover whole cache lines; the sum of squares crosses
// lanes in fp32.
#include "kernels.h"

namespace vla {
namespace {

template <int DH, bool F32>
__device__ __forceinline__ f32x4 load4(const void* p, int64_t at) {
  if constexpr (F32) {
    return *(const f32x4*)((const float*)p + at);
  } else {
    const u32x2 w = *(const u32x2*)((const bf16_t*)p + at);
    return f32x4{__uint_as_float(w[0] << 16), __uint_as_float(w[0] & 0xffff0000u), __uint_as_float(w[1] << 16),
                 __uint_as_float(w[1] & 0xffff0000u)};
  }
}

// one token per workgroup; the 256 threads take its query and key heads in turn
template <int DH, bool F32>
__global__ __launch_bounds__(256) void qk_norm_rope_kernel(QkNormArgs a) {
  constexpr int LN = DH / 8, ROWS = 256 / LN;
  const int tid = threadIdx.x, j = tid % LN, slot = tid / LN;
  const int b = blockIdx.x / a.L, t = blockIdx.x % a.L;
  f32x4 c = {1.f, 1.f, 1.f, 1.f}, s = {0.f, 0.f, 0.f, 0.f};
  if (a.cos) {
    const int pos = a.pos ? a.pos[blockIdx.x] : t;
    if (pos < 0 || pos >= a.n_pos) return;
    c = *(const f32x4*)(a.cos + (size_t)pos * (DH / 2) + 4 * j);
    s = *(const f32x4*)(a.sin + (size_t)pos * (DH / 2) + 4 * j);
  }
  for (int h = slot; h < a.H + a.Hkv; h += ROWS) {
    const bool isq = h < a.H;
    const Heads& in = isq ? a.q : a.k;
    const Heads& out = isq ? a.q_out : a.k_out;
    const float* g = isq ? a.gq : a.gk;
    const int hh = isq ? h : h - a.H;
    const int64_t at = b * in.seq + t * in.token + hh * in.head + 4 * j;
    f32x4 x = load4<DH, F32>(in.p, at), y = load4<DH, F32>(in.p, at + DH / 2);
    if (g) {
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) sum += x[e] * x[e] + y[e] * y[e];
#pragma unroll
      for (int o = 1; o < LN; o <<= 1) sum += __shfl_xor(sum, o);
      const float r = 1.f / sqrtf(sum / DH + a.eps);
      const f32x4 gx = *(const f32x4*)(g + 4 * j), gy = *(const f32x4*)(g + DH / 2 + 4 * j);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[e] = x[e] * r * gx[e];
        y[e] = y[e] * r * gy[e];
      }
    }
    float u[4], v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      u[e] = x[e] * c[e] - y[e] * s[e];
      v[e] = y[e] * c[e] + x[e] * s[e];
    }
    bf16_t* o = (bf16_t*)out.p + b * out.seq + t * out.token + hh * out.head + 4 * j;
    *(u32x2*)o = u32x2{pack_bf2(u[0], u[1]), pack_bf2(u[2], u[3])};
    *(u32x2*)(o + DH / 2) = u32x2{pack_bf2(v[0], v[1]), pack_bf2(v[2], v[3])};
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

hipError_t qk_norm_rope(const QkNormArgs& a, bool f32, int dh, hipStream_t s) {
  return dh == 128 ? launch<128>(a, f32, s) : launch<64>(a, f32, s);
}

}  // namespace vla
