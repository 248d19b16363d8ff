// Products of a few activation rows with 4-bit weights:
//   y[m][n] = sum_k x[m][k] s[n][k/g] (c[n][k] - z[n][k/g])
// c = 0..15, one scale s and zero point z (both bf16) per row and group of g
// = 32, 64 or 128 inputs.
//
// A decode step's product reads every weight once for one to sixteen rows of
// x, so its cost is the stream of the weights.  What has to stay cheap is
// turning codes into operands.  Two VALU instructions make two of them: code
// c shifted to bits 3..6 of a bf16 whose exponent is that of 16 is the exact
// number 16 + c, so
//   sum_k (c - z) x = sum_k (16 + c) x - (16 + z) sum_k x
// within a group.  The first sum is an MFMA (16 rows of x against 16 rows of
// W, 32 k a step), and so is the second, against a matrix of ones: its result
// lies in the lane that needs it.  Scale and zero point then cost two fused
// multiply-adds per accumulator and group, in fp32.  16 is the smallest such
// offset, which keeps the two sums' cancellation to the size of a rounding
// of fp32 (with 128, the exponent at which codes need no shift, it would be
// eight times that).
//
// Rows of x sit in the accumulator rows that one register of the MFMA result
// covers: with M <= 4 in rows 0, 4, 8, 12, so a lane holds one useful value
// (R = 1) and scales that alone; M <= 8 uses two (R = 2), up to 16 all four.
#include "kernels.h"

namespace vla {
namespace {

// The packed weights: rows in tiles of 16, k in blocks of 128.
//   codes  [tile][block][lane 64][4] 32-bit words: lane l holds row l % 16; its
//          word t the 8 codes k = 32 t + 8 (l / 16) + j of the block, code j
//          in nibble j / 2 (even j) or 4 + j / 2 (odd j)
//   params [tile][block][row 16][128 / g] 32-bit words: scale in the low,
//          zero point in the high half
// Rows past N and inputs past K have code 0 and scale 0.
__host__ __device__ inline size_t code_bytes(int N, int K) { return (size_t)cdiv(N, 16) * cdiv(K, 128) * 1024; }

constexpr uint32_t BIAS16 = 0x41804180u;  // bf16 16.0 twice
constexpr uint32_t CODE_BITS = 0x00780078u;

// 8 codes of a word as bf16 numbers 16 + c
__device__ __forceinline__ bf16x8 unpack8(uint32_t w) {
  const u32x4 v = {(w << 3 & CODE_BITS) | BIAS16, (w >> 1 & CODE_BITS) | BIAS16, (w >> 5 & CODE_BITS) | BIAS16,
                   (w >> 9 & CODE_BITS) | BIAS16};
  return __builtin_bit_cast(bf16x8, v);
}

__device__ __forceinline__ f32x4 mfma(const bf16x8& a, const bf16x8& b, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

struct W4Args {
  const bf16_t* x;
  int64_t ldx;
  const uint8_t* wp;
  const float* res;
  void* out;
  int64_t ldo;
  int M, N, K;
};

// One workgroup: NT tiles of 16 weight rows (SWIGLU: NT / 2 gate tiles and
// the up tiles of the same features), 16 rows of x; its W waves take every
// W-th block of 128 k and join their sums in LDS.
template <int NT, int R, int GPB, int W, bool SWIGLU, bool F32>
__global__ __launch_bounds__(W * 64) void w4_kernel(W4Args a) {
  __shared__ float red[W][NT * R][64];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c16 = lane & 15, kq = lane >> 4;
  const int ntiles = cdiv(a.N, 16), KB = cdiv(a.K, 128);
  constexpr int TW = SWIGLU ? NT / 2 : NT;  // output tiles
  const int t0 = blockIdx.x * TW;
  const int m0 = blockIdx.y * 16;
  int tile[NT];
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    const int t = SWIGLU ? (i < TW ? min(t0 + i, ntiles / 2 - 1) : ntiles / 2 + min(t0 + i - TW, ntiles / 2 - 1))
                         : min(t0 + i, ntiles - 1);
    tile[i] = t;
  }
  // x rows: MFMA row c16 = 4 i + r holds row i R + r (r < R); others and rows
  // past M read as zero
  const int m = (c16 >> 2) * R + (c16 & 3);
  const bool row_there = (c16 & 3) < R && m0 + m < a.M;
  const bf16_t* xrow = a.x + (size_t)(row_there ? m0 + m : 0) * a.ldx;
  const uint8_t* pp = a.wp + code_bytes(a.N, a.K);
  const bf16x8 ones = __builtin_bit_cast(bf16x8, u32x4{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u});
  float y[NT][R];
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int r = 0; r < R; ++r) y[i][r] = 0.f;

  for (int kb = wave; kb < KB; kb += W) {
    u32x4 cw[NT];
    uint32_t pw[NT][GPB];
    bf16x8 xa[4];
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      cw[i] = *(const u32x4*)(a.wp + ((size_t)tile[i] * KB + kb) * 1024 + lane * 16);
      const uint32_t* p = (const uint32_t*)pp + (((size_t)tile[i] * KB + kb) * 16 + c16) * GPB;
#pragma unroll
      for (int g = 0; g < GPB; ++g) pw[i][g] = p[g];
    }
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int k = kb * 128 + t * 32 + kq * 8;
      u32x4 v = {0u, 0u, 0u, 0u};
      if (row_there && k < a.K) v = *(const u32x4*)(xrow + k);
      xa[t] = __builtin_bit_cast(bf16x8, v);
    }
#pragma unroll
    for (int g = 0; g < GPB; ++g) {
      f32x4 xs = {0.f, 0.f, 0.f, 0.f}, d[NT];
#pragma unroll
      for (int i = 0; i < NT; ++i) d[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int t = g * 4 / GPB; t < (g + 1) * 4 / GPB; ++t) {
        xs = mfma(xa[t], ones, xs);
#pragma unroll
        for (int i = 0; i < NT; ++i) d[i] = mfma(xa[t], unpack8(cw[i][t]), d[i]);
      }
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        const float s = __uint_as_float(pw[i][g] << 16), z = __uint_as_float(pw[i][g] & 0xffff0000u);
#pragma unroll
        for (int r = 0; r < R; ++r) y[i][r] = fmaf(s, fmaf(-16.f - z, xs[r], d[i][r]), y[i][r]);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int r = 0; r < R; ++r) red[wave][i * R + r][lane] = y[i][r];
  __syncthreads();
  for (int e = wave; e < TW * R; e += W) {
    const int i = e / R, r = e % R;
    float v = 0.f, u = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) v += red[w][e][lane];
    if constexpr (SWIGLU) {
#pragma unroll
      for (int w = 0; w < W; ++w) u += red[w][TW * R + e][lane];
    }
    const int n = (t0 + i) * 16 + c16, row = m0 + kq * R + r;
    if (n < (SWIGLU ? a.N / 2 : a.N) && row < a.M) {
      if constexpr (SWIGLU) v = v / (1.f + __expf(-v)) * u;
      const size_t at = (size_t)row * a.ldo + n;
      if (a.res) v += a.res[at];
      if constexpr (F32)
        ((float*)a.out)[at] = v;
      else
        ((bf16_t*)a.out)[at] = f2bf(v);
    }
  }
}

template <int NT, int R, int W, bool SWIGLU, bool F32>
hipError_t launch(const W4Args& a, int group, hipStream_t s) {
  const int tiles = SWIGLU ? a.N / 32 : cdiv(a.N, 16), tw = SWIGLU ? NT / 2 : NT;
  const dim3 grid(cdiv(tiles, tw), cdiv(a.M, 16)), block(W * 64);
  switch (group) {
    case 32: hipLaunchKernelGGL((w4_kernel<NT, R, 4, W, SWIGLU, F32>), grid, block, 0, s, a); break;
    case 64: hipLaunchKernelGGL((w4_kernel<NT, R, 2, W, SWIGLU, F32>), grid, block, 0, s, a); break;
    default: hipLaunchKernelGGL((w4_kernel<NT, R, 1, W, SWIGLU, F32>), grid, block, 0, s, a); break;
  }
  return hipGetLastError();
}

template <bool SWIGLU, bool F32>
hipError_t by_rows(const W4Args& a, int group, hipStream_t s) {
  constexpr int NT = SWIGLU ? 2 : 1;
  if (a.M <= 4) return launch<NT, 1, 8, SWIGLU, F32>(a, group, s);
  if (a.M <= 8) return launch<NT, 2, 8, SWIGLU, F32>(a, group, s);
  return launch<NT, 4, 8, SWIGLU, F32>(a, group, s);
}

// one thread per word of the packed weights
__global__ __launch_bounds__(256) void w4_pack_kernel(const uint8_t* __restrict__ codes,
                                                      const bf16_t* __restrict__ scales,
                                                      const bf16_t* __restrict__ zeros, uint32_t* __restrict__ wp, int N,
                                                      int K, int group) {
  const int KB = cdiv(K, 128), G = cdiv(K, group), gpb = 128 / group;
  const size_t nc = code_bytes(N, K) / 4, np = (size_t)cdiv(N, 16) * KB * 16 * gpb;
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < nc + np; i += (size_t)gridDim.x * 256) {
    uint32_t w = 0;
    if (i < nc) {
      const int t = (int)(i % 4), lane = (int)(i / 4 % 64);
      const size_t blk = i / 256;
      const int n = (int)(blk / KB) * 16 + lane % 16, k = (int)(blk % KB) * 128 + t * 32 + lane / 16 * 8;
      if (n < N)
        for (int j = 0; j < 8; ++j)
          if (k + j < K) w |= (uint32_t)(codes[(size_t)n * K + k + j] & 15) << 4 * (j / 2 + (j & 1) * 4);
    } else {
      const size_t q = i - nc;
      const int g = (int)(q % gpb), r = (int)(q / gpb % 16);
      const size_t blk = q / gpb / 16;
      const int n = (int)(blk / KB) * 16 + r, gg = (int)(blk % KB) * gpb + g;
      if (n < N && gg < G) {
        const uint32_t z = zeros ? zeros[(size_t)n * G + gg] : 0x4100u;  // 8
        w = scales[(size_t)n * G + gg] | z << 16;
      }
    }
    wp[i] = w;
  }
}

}  // namespace

size_t w4_packed_bytes(int N, int K, int group) {
  return code_bytes(N, K) + (size_t)cdiv(N, 16) * cdiv(K, 128) * 16 * (128 / group) * 4;
}

hipError_t w4_pack(const uint8_t* codes, const bf16_t* scales, const bf16_t* zeros, void* wp, int N, int K, int group,
                   hipStream_t s) {
  const size_t words = w4_packed_bytes(N, K, group) / 4;
  const unsigned grid = (unsigned)((words + 255) / 256 < 65536 ? (words + 255) / 256 : 65536);
  hipLaunchKernelGGL(w4_pack_kernel, dim3(grid), dim3(256), 0, s, codes, scales, zeros, (uint32_t*)wp, N, K, group);
  return hipGetLastError();
}

hipError_t gemv_w4(const bf16_t* x, int64_t ldx, const void* wp, const float* res, void* out, int64_t ldo, bool f32,
                   bool swiglu, int M, int N, int K, int group, hipStream_t s) {
  const W4Args a{x, ldx, (const uint8_t*)wp, res, out, ldo, M, N, K};
  if (swiglu) return f32 ? by_rows<true, true>(a, group, s) : by_rows<true, false>(a, group, s);
  return f32 ? by_rows<false, true>(a, group, s) : by_rows<false, false>(a, group, s);
}

}  // namespace vla
