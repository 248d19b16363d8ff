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
// That leaves 7 instructions and an MFMA for the 512 weights of a word a lane, so
// the stream of weights is the bound where it is long, us from the 256 MB cache
// (three calls' weights in turn) and from memory (1.3 GB in turn, as the layers of
// a decode step read them; 2.3 are a launch's own):
//   26 MB, N = 12288, K = 4096, one row:  6.4, 7.2
//   48 MB, gated, 2 x 11008, K = 4096, four rows:  10.0, 12.0
//   29 MB, N = 4096, K = 11008, 13 rows:  8.7, 12.3
// The last has 256 workgroups of six blocks of k in a row for each wave, and a
// block from memory takes longer.  More than 16 rows read the weights once per 16:
// N = 12288, K = 4096, 64 rows 16 us, 256 rows 52 (the bf16 product of 256 rows: 31).
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
//          in nibble j / 2 (even j) or 4 + j / 2 (odd j), the word rotated
//          left by 3: nibbles i and 4 + i, 4 i bits to the right, are then the
//          top mantissa bits of a pair
//   params [tile][block][row 16][128 / g] 32-bit words: scale in the low,
//          zero point in the high half
// Rows past N and inputs past K have code 0 and scale 0.
__host__ __device__ inline size_t code_bytes(int N, int K) { return (size_t)cdiv(N, 16) * cdiv(K, 128) * 1024; }

constexpr int ROT = 3;

struct W4Args {
  const bf16_t* x;
  int64_t ldx;
  const uint8_t* wp;
  const float* res;
  void* out;
  int64_t ldo;
  int M, N, K;
  bool f32;
};

template <int N>
struct alignas(4 * N) Params {
  uint32_t w[N];
};

// One workgroup: NT tiles of 16 weight rows (SWIGLU: NT / 2 gate tiles and
// the up tiles of the same features), 16 rows of x; its W waves take every
// W-th block of 128 k and join their sums in LDS.
template <int NT, int R, int GPB, int W, bool SWIGLU>
__global__ __launch_bounds__(W * 64) void w4_kernel(W4Args a) {
  // a wave's block of x, then its sums
  constexpr int XW = 4 * R * 16, SW = NT * R * 16;  // 16-byte words
  __shared__ u32x4 lds[W][XW > SW ? XW : SW];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c16 = lane & 15, kq = lane >> 4;
  const int ntiles = cdiv(a.N, 16), KB = cdiv(a.K, 128);
  constexpr int TW = SWIGLU ? NT / 2 : NT;  // output tiles
  const int t0 = blockIdx.x * TW;
  const int m0 = blockIdx.y * 16;
  const uint8_t* codes[NT];
  const uint8_t* params[NT];
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    const int t = SWIGLU ? (i < TW ? min(t0 + i, ntiles / 2 - 1) : ntiles / 2 + min(t0 + i - TW, ntiles / 2 - 1))
                         : min(t0 + i, ntiles - 1);
    codes[i] = a.wp + (size_t)t * KB * 1024;
    params[i] = a.wp + code_bytes(a.N, a.K) + (size_t)t * KB * (64 * GPB);
  }
  const int mrows = min(a.M - m0, 16);
  const __amdgpu_buffer_rsrc_t xr = __builtin_amdgcn_make_buffer_rsrc(
      (void*)(a.x + (size_t)m0 * a.ldx), (short)0, (int)(((size_t)(mrows - 1) * a.ldx + a.K) * 2), 0x00020000);
  const UnpackCodes unpack;
  const bf16x8 ones = __builtin_bit_cast(bf16x8, u32x4{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u});
  float y[NT][R];
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int r = 0; r < R; ++r) y[i][r] = 0.f;

  // x: load q covers rows 4 q .. 4 q + 3, 16 lanes and 256 bytes each (a lane
  // per operand word would touch 16 rows in 16-byte pieces, and the gather cost
  // more than the weights at 16 rows); rows and inputs that are not there lie
  // outside the buffer and read as zero.  LDS turns them into operands: MFMA row
  // 4 i + r is row i R + r (r < R; the others repeat one, their results are not
  // used); word c of row m lies at c ^ 4 (m & 3), free of bank conflicts.
  u32x4* xs = lds[wave];
  uint32_t xat[R];
#pragma unroll
  for (int q = 0; q < R; ++q) {
    const int row = 4 * q + kq;
    xat[q] = row < mrows ? (uint32_t)(row * a.ldx * 2) + c16 * 16 : 0x80000000u;
  }
  const int xput = kq * 16 + (c16 ^ kq * 4);
  const int xrow = (c16 >> 2) * R + min(c16 & 3, R - 1), xget = xrow * 16, xswz = (xrow & 3) * 4;

  // a block's registers, loaded again as soon as they are used up, in parts.  Past
  // the last block the buffers are empty and the loads touch no memory: with a
  // branch around them, with uses of the old values below them or with the first
  // loads in another order than the loop's, the compiler waits for every load at
  // the loop's end (2 to 8% of the time).  A second block ahead costs waves: 6.5 ->
  // 7.0 us at N = 12288, K = 4096, one row.
  u32x4 xw[R], cw[NT];
  Params<GPB> pw[NT];
  // x of 16 rows is 16 registers, and asked for after the codes (N = 4096, K = 11008,
  // 13 rows: 8.6 us, before them 9.2)
  constexpr bool LATE_X = R == 4;
  auto fetch_x = [&](int kb) {
    const bool in = kb * 128 + c16 * 8 < a.K;
#pragma unroll
    for (int q = 0; q < R; ++q)
      xw[q] = __builtin_bit_cast(
          u32x4, __builtin_amdgcn_raw_buffer_load_b128(xr, in ? xat[q] + kb * 256 : 0x80000000u, 0, 0));
  };
  auto fetch_codes = [&](int kb) {
#pragma unroll
    for (int i = 0; i < NT; ++i)
      cw[i] = __builtin_bit_cast(
          u32x4, __builtin_amdgcn_raw_buffer_load_b128(
                     __builtin_amdgcn_make_buffer_rsrc((void*)codes[i], (short)0, kb < KB ? KB * 1024 : 0, 0x00020000),
                     lane * 16, kb < KB ? kb * 1024 : 0, 0));
  };
  auto fetch_params = [&](int kb) {
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(
          (void*)params[i], (short)0, kb < KB ? KB * (64 * GPB) : 0, 0x00020000);
      const uint32_t at = c16 * (4 * GPB), base = kb < KB ? kb * (64 * GPB) : 0;
      if constexpr (GPB == 1)
        pw[i].w[0] = __builtin_amdgcn_raw_buffer_load_b32(r, at, base, 0);
      else if constexpr (GPB == 2)
        pw[i] = __builtin_bit_cast(Params<2>, __builtin_amdgcn_raw_buffer_load_b64(r, at, base, 0));
      else
        pw[i] = __builtin_bit_cast(Params<4>, __builtin_amdgcn_raw_buffer_load_b128(r, at, base, 0));
    }
  };
  if (!LATE_X) fetch_x(wave);
  __builtin_amdgcn_sched_barrier(0);
  fetch_codes(wave);
  __builtin_amdgcn_sched_barrier(0);
  if (LATE_X) fetch_x(wave);
  __builtin_amdgcn_sched_barrier(0);
  fetch_params(wave);
  __builtin_amdgcn_sched_barrier(0);
  for (int kb = wave; kb < KB; kb += W) {
#pragma unroll
    for (int q = 0; q < R; ++q) xs[q * 64 + xput] = xw[q];
    __builtin_amdgcn_sched_barrier(0);
    if (!LATE_X) fetch_x(kb + W);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    bf16x8 xa[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) xa[t] = __builtin_bit_cast(bf16x8, xs[xget + ((t * 4 + kq) ^ xswz)]);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    f32x4 sum[GPB], d[GPB][NT];
#pragma unroll
    for (int g = 0; g < GPB; ++g) {
      sum[g] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < NT; ++i) d[g][i] = sum[g];
#pragma unroll
      for (int t = g * 4 / GPB; t < (g + 1) * 4 / GPB; ++t) {
        sum[g] = mfma(xa[t], ones, sum[g]);
#pragma unroll
        for (int i = 0; i < NT; ++i) d[g][i] = mfma(xa[t], unpack(cw[i][t]), d[g][i]);
      }
    }
    // keeps the unused rows' registers from being used again before the MFMAs are done
#pragma unroll
    for (int g = 0; g < GPB; ++g) {
      asm volatile("" : "+v"(sum[g]));
#pragma unroll
      for (int i = 0; i < NT; ++i) asm volatile("" : "+v"(d[g][i]));
    }
    __builtin_amdgcn_sched_barrier(0);
    fetch_codes(kb + W);
    __builtin_amdgcn_sched_barrier(0);
    if (LATE_X) fetch_x(kb + W);
#pragma unroll
    for (int g = 0; g < GPB; ++g)
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        const uint32_t p = pw[i].w[g];
        const float s = __uint_as_float(p << 16), z = __uint_as_float(p & 0xffff0000u);
#pragma unroll
        for (int r = 0; r < R; ++r) y[i][r] = fmaf(s, fmaf(-16.f - z, sum[g][r], d[g][i][r]), y[i][r]);
      }
    __builtin_amdgcn_sched_barrier(0);
    fetch_params(kb + W);
  }
  float* red = (float*)lds[wave];
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int r = 0; r < R; ++r) red[(i * R + r) * 64 + lane] = y[i][r];
  __syncthreads();
  for (int e = wave; e < TW * R; e += W) {
    const int i = e / R, r = e % R;
    float v = 0.f, u = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) v += ((const float*)lds[w])[e * 64 + lane];
    if constexpr (SWIGLU) {
#pragma unroll
      for (int w = 0; w < W; ++w) u += ((const float*)lds[w])[(TW * R + e) * 64 + lane];
    }
    const int n = (t0 + i) * 16 + c16, row = m0 + kq * R + r;
    if (n < (SWIGLU ? a.N / 2 : a.N) && row < a.M) {
      if constexpr (SWIGLU) v = v / (1.f + __expf(-v)) * u;
      const size_t at = (size_t)row * a.ldo + n;
      if (a.res) v += a.res[at];
      if (a.f32)
        ((float*)a.out)[at] = v;
      else
        ((bf16_t*)a.out)[at] = f2bf(v);
    }
  }
}

template <int NT, int R, int W, bool SWIGLU>
hipError_t launch(const W4Args& a, int group, hipStream_t s) {
  const int tiles = SWIGLU ? a.N / 32 : cdiv(a.N, 16), tw = SWIGLU ? NT / 2 : NT;
  const dim3 grid(cdiv(tiles, tw), cdiv(a.M, 16)), block(W * 64);
  switch (group) {
    case 32: hipLaunchKernelGGL((w4_kernel<NT, R, 4, W, SWIGLU>), grid, block, 0, s, a); break;
    case 64: hipLaunchKernelGGL((w4_kernel<NT, R, 2, W, SWIGLU>), grid, block, 0, s, a); break;
    default: hipLaunchKernelGGL((w4_kernel<NT, R, 1, W, SWIGLU>), grid, block, 0, s, a); break;
  }
  return hipGetLastError();
}

template <int NT, int W>
hipError_t by_rows(const W4Args& a, int group, bool swiglu, hipStream_t s) {
  if constexpr (NT > 1) {
    if (swiglu)
      return a.M <= 4   ? launch<NT, 1, W, true>(a, group, s)
             : a.M <= 8 ? launch<NT, 2, W, true>(a, group, s)
                        : launch<NT, 4, W, true>(a, group, s);
  }
  return a.M <= 4   ? launch<NT, 1, W, false>(a, group, s)
         : a.M <= 8 ? launch<NT, 2, W, false>(a, group, s)
                    : launch<NT, 4, W, false>(a, group, s);
}

// Tiles and waves a workgroup, by the estimated time of each choice, in
// hundredths of a microsecond: a wave takes 70 a block of 128 k and 7 more a tile,
// a SIMD 12 a tile and block, 9 a block for x past four rows and 18 a wave; one CU
// takes the workgroups past 256; a tile costs 37 at the ends.  More waves shorten
// each one's chain of blocks, more tiles share the turning of x into operands, and
// both leave fewer workgroups.  Over 332 calls timed at every choice (N = 1024 to
// 57344, K = 896 to 16384, 1 to 13 rows, plain and gated) what this takes is 0.6%
// slower than the fastest on average and 9% at most, and over 110 others, drawn
// from N = 32 to 160000 and K = 64 to 32768, 0.5% and 7%.  us, tiles x waves:
//   N = 4096, K = 16384, 13 rows, g = 128:  1 x 8 10.4, 1 x 16 9.6
//   N = 8192, K = 8192, 13 rows, g = 32:  1 x 8 11.0, 2 x 16 9.9
//   N = 28672, K = 8192, 13 rows, g = 128:  1 x 4 39.6, 4 x 4 26.4
//   N = 57344, K = 8192, one row:  1 x 8 46.7, 2 x 16 39.7; seven 1 x 4 66, 2 x 8 49
struct Shape {
  int tiles, waves;
};
Shape shape_of(int M, int N, int K, bool swiglu) {
  Shape best{};
  int64_t least = INT64_MAX;
  for (int n = swiglu ? 2 : 1; n <= 4; n *= 2)
    for (int w = 4; w <= (n < 4 ? 16 : 8); w *= 2) {
      const int64_t wgs = (int64_t)cdiv(cdiv(N, 16), n) * cdiv(M, 16), per = cdiv(cdiv(K, 128), w);
      const int64_t chain = per * (70 + 7 * n), simd = (wgs + 255) / 256 * (w / 4) * (per * ((M > 4 ? 9 : 0) + 12 * n) + 18);
      const int64_t cost = (chain > simd ? chain : simd) + 37 * n;
      if (cost < least) least = cost, best = Shape{n, w};
    }
  return best;
}

// One thread per word of the packed weights, whose 8 codes are bytes of one row;
// neighbours in a wave take rows K apart.  Once a matrix, at load: N = 12288, K =
// 4096 (50 MB of codes, 27 packed) 87 us, 0.9 TB/s.
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
    wp[i] = i < nc ? rotl(w, ROT) : w;
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
  const W4Args a{x, ldx, (const uint8_t*)wp, res, out, ldo, M, N, K, f32};
  const Shape h = shape_of(M, N, K, swiglu);
  if (h.tiles == 4) return h.waves == 8 ? by_rows<4, 8>(a, group, swiglu, s) : by_rows<4, 4>(a, group, swiglu, s);
  if (h.tiles == 2)
    return h.waves == 16  ? by_rows<2, 16>(a, group, swiglu, s)
           : h.waves == 8 ? by_rows<2, 8>(a, group, swiglu, s)
                          : by_rows<2, 4>(a, group, swiglu, s);
  return h.waves == 16  ? by_rows<1, 16>(a, group, false, s)
         : h.waves == 8 ? by_rows<1, 8>(a, group, false, s)
                        : by_rows<1, 4>(a, group, false, s);
}

}  // namespace vla
