// Products of int8 rows with int8 weights, a scale a row of each:
//   y[m][n] = sx[m] sw[n] sum_k x[m][k] w[n][k]
// the sum by v_mfma_i32_16x16x64_i8 in 32-bit whole numbers, which hold it exactly
// (K <= 131056): its order does not matter, so K may be dealt out to waves as suits.
// The accumulator is converted once and scaled in fp32.
//
// The packed weights are MFMA operands in the order in which lanes take them: tiles
// of 16 rows, k in steps of 64, each (tile, step) 1024 contiguous bytes, lane l's 16
// codes k = 64 step + 16 (l / 16) + j of row l % 16 at byte 16 l; a tile's steps lie
// side by side, a multiple of four of them, zeros past K and N.  (What x holds there
// is multiplied by zero: rows of x are read as they lie, past their end the next one.)  Rows are dealt to two
// tiles at a time: row 4 q + r of the tile pair's first tile is row 8 q + r of its 32,
// of its second tile 8 q + 4 + r.  So a lane's accumulators, rows 4 q + r of one x
// row, are 8 outputs side by side over a pair.  The scales follow, one a row, in the
// same order.
#include <type_traits>

#include "kernels.h"

namespace vla {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

__host__ __device__ inline int tiles_of(int N) { return (N + 31) / 32 * 2; }
__host__ __device__ inline int steps_of(int K) { return (K + 255) / 256 * 4; }
__host__ __device__ inline size_t code_bytes(int N, int K) { return (size_t)tiles_of(N) * steps_of(K) * 1024; }
// row of W that lies in row r of tile t
__host__ __device__ inline int row_of(int t, int r) { return (t >> 1) * 32 + (r >> 2) * 8 + (t & 1) * 4 + (r & 3); }

__device__ __forceinline__ i32x4 mfma_i8(const i32x4& a, const i32x4& b, const i32x4& c) {
  return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ float silu_of(float g) { return g / (1.f + __expf(-g)); }

// What a buffer's range check must cut is in the vector offset or in the buffer's own start and size; scalar offsets are 0
// throughout, since a check need not count them.

// Rows [m0, m0 + rows) of out and of the residual as buffers: a store past them, or one
// to NOWHERE, is dropped, so the epilogue has no branches.  WIDE: four outputs side by
// side exist together, and rows are aligned for them.
constexpr uint32_t NOWHERE = 0x80000000u;
template <bool WIDE, bool F32>
struct Rows {
  __amdgpu_buffer_rsrc_t out, res;
  int N;
  __device__ __forceinline__ Rows(const GemmI8Args& a, int m0, int rows, int n) : N(n) {
    const int64_t elems = (rows - 1) * a.ldo + n;
    out = __builtin_amdgcn_make_buffer_rsrc((uint8_t*)a.out + m0 * a.ldo * (F32 ? 4 : 2), (short)0,
                                            (int)(elems * (F32 ? 4 : 2)), 0x00020000);
    res = __builtin_amdgcn_make_buffer_rsrc((void*)(a.res + (a.res ? m0 * a.ldo : 0)), (short)0,
                                            a.res ? (int)(elems * 4) : 0, 0x00020000);
  }
  // columns col .. col + 3, element `at` of these rows (where `in`)
  __device__ __forceinline__ f32x4 residual(uint32_t at, int col, bool in) const {
    if constexpr (WIDE)
      return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(res, in && col < N ? at * 4 : NOWHERE, 0, 0));
    f32x4 r;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      r[e] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(res, in && col + e < N ? (at + e) * 4 : NOWHERE, 0, 0));
    return r;
  }
  __device__ __forceinline__ void store(uint32_t at, int col, bool in, const f32x4& v) const {
    if constexpr (WIDE) {
      const uint32_t to = in && col < N ? at * (F32 ? 4 : 2) : NOWHERE;
      if constexpr (F32)
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), out, to, 0, 0);
      else
        __builtin_amdgcn_raw_buffer_store_b64(u32x2{pack_bf2(v[0], v[1]), pack_bf2(v[2], v[3])}, out, to, 0, 0);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x = v[e];
        if constexpr (F32)
          __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(x), out, in && col + e < N ? (at + e) * 4 : NOWHERE, 0, 0);
        else
          __builtin_amdgcn_raw_buffer_store_b16(f2bf(x), out, in && col + e < N ? (at + e) * 2 : NOWHERE, 0, 0);
      }
    }
  }
};
// f(wide, f32) with the call's own as constants
template <class F>
__device__ __forceinline__ void by_output(const GemmI8Args& a, F f) {
  if (a.wide) {
    if (a.f32)
      f(std::true_type{}, std::true_type{});
    else
      f(std::true_type{}, std::false_type{});
  } else {
    if (a.f32)
      f(std::false_type{}, std::true_type{});
    else
      f(std::false_type{}, std::false_type{});
  }
}

// ------------------------------------------------------------------ few rows
//
// Up to 16 rows of x: the weights' bytes are the bound.  A workgroup takes NT tiles of
// weight rows (SWIGLU: NT / 2 gate tiles and the up tiles of the same features); its W
// waves take runs of U steps in turn and add up in LDS.  Weights and x go from memory
// into registers, a run ahead.  One row, 12288 x 4096: 9.6 us, 11.7 with the weights
// from memory (5.4 TB/s behind the launch's 2.3 us).
template <int NT, int W, int U, bool SWIGLU>
__global__ __launch_bounds__(W * 64) void w8_rows_kernel(GemmI8Args a) {
  __shared__ i32x4 part[W][NT][64];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c16 = lane & 15, q = lane >> 4;
  const int KS = steps_of(a.K), ntiles = tiles_of(a.N), half = ntiles / 2;
  constexpr int TW = SWIGLU ? NT / 2 : NT;
  const int t0 = blockIdx.x * TW;
  const uint8_t* wt[NT];
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    const int t = SWIGLU ? (i < TW ? min(t0 + i, half - 1) : half + min(t0 + i - TW, half - 1)) : min(t0 + i, ntiles - 1);
    wt[i] = a.wp + (size_t)t * KS * 1024;
  }
  // past the row of x: its next one, or zeros past the last; the weights there are zero
  const int xbytes = (int)((a.M - 1) * a.ldx + a.K);
  const uint32_t xat = c16 < a.M ? (uint32_t)(c16 * a.ldx) + q * 16 : NOWHERE;
  i32x4 wr[2][NT][U], xr[2][U];
  auto fetch = [&](int b, int s0) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool in = s0 + u < KS;  // past the last step: empty buffers, no memory is touched
#pragma unroll
      for (int i = 0; i < NT; ++i)
        wr[b][i][u] = __builtin_bit_cast(
            i32x4, __builtin_amdgcn_raw_buffer_load_b128(
                       __builtin_amdgcn_make_buffer_rsrc((void*)(wt[i] + (s0 + u) * 1024), (short)0, in ? 1024 : 0, 0x00020000),
                       lane * 16, 0, 0));
      const int k = (s0 + u) * 64;  // may lie past the row's end, where the weights' steps are padded
      xr[b][u] = __builtin_bit_cast(
          i32x4, __builtin_amdgcn_raw_buffer_load_b128(
                     __builtin_amdgcn_make_buffer_rsrc((void*)(a.x + k), (short)0, in ? max(xbytes - k, 0) : 0, 0x00020000),
                     xat, 0, 0));
    }
  };
  i32x4 acc[NT];
#pragma unroll
  for (int i = 0; i < NT; ++i) acc[i] = i32x4{0, 0, 0, 0};
  auto multiply = [&](int b) {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < NT; ++i) acc[i] = mfma_i8(wr[b][i][u], xr[b][u], acc[i]);
  };
  int s = wave * U;
  fetch(0, s);
  while (s < KS) {
    fetch(1, s + W * U);
    __builtin_amdgcn_sched_barrier(0);
    multiply(0);
    s += W * U;
    if (s >= KS) break;
    fetch(0, s + W * U);
    __builtin_amdgcn_sched_barrier(0);
    multiply(1);
    s += W * U;
  }
#pragma unroll
  for (int i = 0; i < NT; ++i) part[wave][i][lane] = acc[i];
  __syncthreads();
  const float* sw = (const float*)(a.wp + code_bytes(a.N, a.K));
  const int N = SWIGLU ? a.N / 2 : a.N;
  for (int i = wave; i < TW; i += W) {
    const int t = min(t0 + i, (SWIGLU ? half : ntiles) - 1), col = row_of(t0 + i, 4 * q);
    auto joined = [&](int i) {
      i32x4 v = part[0][i][lane];
#pragma unroll
      for (int w = 1; w < W; ++w) v += part[w][i][lane];
      return v;
    };
    const i32x4 v = joined(i), u = SWIGLU ? joined(i + TW) : v;
    const float sx = a.sx[min(c16, a.M - 1)];
    const f32x4 ws = *(const f32x4*)(sw + t * 16 + q * 4);
    f32x4 y;
#pragma unroll
    for (int x = 0; x < 4; ++x) y[x] = (float)v[x] * sx * ws[x];
    if constexpr (SWIGLU) {
      const f32x4 us = *(const f32x4*)(sw + (half + t) * 16 + q * 4);
#pragma unroll
      for (int x = 0; x < 4; ++x) y[x] = silu_of(y[x]) * ((float)u[x] * sx * us[x]);
    }
    by_output(a, [&](auto wide, auto f32) {
      const Rows<wide.value, f32.value> io(a, 0, a.M, N);
      const uint32_t at = c16 * (uint32_t)a.ldo + col;
      if (a.res) y += io.residual(at, col, c16 < a.M);
      io.store(at, col, c16 < a.M, y);
    });
  }
}

// ----------------------------------------------------------------- many rows
//
// A workgroup of WGN KG waves takes BM rows of x by BN rows of W, each wave all BM rows by
// BN / WGN (KG = 2: two waves of them, one for the even steps of 64 k and one for the odd
// ones, joined in LDS at the end).  Weights go from memory straight into the registers of the
// one wave that multiplies them, D steps ahead.  x goes to LDS by buffer_load ... lds, two
// steps (a slab) at a time into a ring of NX, and is read LA operands ahead of the
// MFMAs that take it, so a slab costs one barrier.
//
// What bounds it is how fast a CU is filled, 70 GB/s or 33 bytes a cycle in whole cache
// lines: (BM + BN) 64 bytes a step against BM BN / 64 cycles of MFMAs (8192 operations a
// cycle and CU).  With 64 bytes of a row of x a load, in place of the 128 of a cache line,
// x counted twice (333 x 4096, K = 11008 38 us, now 27).
template <int BM, int BN, int WGN, int KG, int NX, int D, int LA, bool SWIGLU>
__global__ __launch_bounds__(64 * WGN * KG) void w8_tile_kernel(GemmI8Args a) {
  constexpr int NW = WGN * KG, TM = BM / 16, TN = BN / WGN / 16, SP = 2 / KG;  // own steps a slab
  constexpr int XB = BM / 8, PX = (XB + NW - 1) / NW, XS = XB * 1024;            // 1 KB loads of a slab of x
  static_assert(PX <= 2, "offsets of a slab's loads");
  static_assert(TM % LA == 0 && D % SP == 0 && (NX - 1) * PX + D * TN < 64, "unrolling, vmcnt range");
  static_assert(!SWIGLU || TN % 2 == 0, "a wave's tiles must be whole (gate, up) pairs");
  constexpr int RED = KG > 1 ? WGN * TM * TN * 1024 : 0;
  __shared__ __attribute__((aligned(1024))) char smem[NX * XS > RED ? NX * XS : RED];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kg = wave / WGN, wn = wave % WGN;
  const int c16 = lane & 15, q = lane >> 4;
  const int KS = steps_of(a.K), ntiles = tiles_of(a.N), half = ntiles / 2;

  // tiles: each of the 8 XCDs takes a contiguous run of them, walked M first inside
  // groups of 8 tile rows
  const int tiles_m = (a.M + BM - 1) / BM, tiles_n = (a.N + BN - 1) / BN;
  int id = blockIdx.x;
  {
    const int per = gridDim.x >> 3, rem = gridDim.x & 7, x = id & 7;
    id = x * per + min(x, rem) + (id >> 3);
  }
  const int group = 8 * tiles_n, first_m = id / group * 8, gsz = min(tiles_m - first_m, 8);
  const int m0 = (first_m + id % group % gsz) * BM, tile_n = id % group / gsz;
  const int rows = min(a.M - m0, BM);

  // x: 8 rows of 128 bytes a load; of 16 rows, row r has its 16-byte chunk c at c ^ (r / 2)
  // of 128, so that 16 rows of one chunk meet every bank alike
  const uint8_t* xp = (const uint8_t*)a.x + (int64_t)m0 * a.ldx;
  const int xbytes = (int)((rows - 1) * a.ldx + a.K);
  uint32_t xvoff[2];
#pragma unroll
  for (int j = 0; j < PX; ++j) {
    const int blk = wave * PX + j;
    xvoff[j] = (uint32_t)((blk * 8 + (lane >> 3)) * a.ldx) + ((lane & 7) ^ (4 * (blk & 1) + (lane >> 4))) * 16;
  }
  auto issue_x = [&](int slab, char* st) {
    // past the last slab: an empty buffer, no memory is touched
    const __amdgpu_buffer_rsrc_t rx = __builtin_amdgcn_make_buffer_rsrc(
        (void*)(xp + slab * 128), (short)0, 2 * slab < KS ? max(xbytes - slab * 128, 0) : 0, 0x00020000);
#pragma unroll
    for (int j = 0; j < PX; ++j) {
      const int blk = wave * PX + j;
      if (PX * NW == XB || blk < XB)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rx, (__attribute__((address_space(3))) void*)(st + blk * 1024), 16,
                                                 xvoff[j], 0, 0, 0);
    }
  };
  // W: SWIGLU takes gate and up tiles of the same features in turn
  const int t0 = SWIGLU ? tile_n * (BN / 32) : tile_n * (BN / 16);  // first tile of W (of the gate's)
  const int wt = min((SWIGLU ? half : ntiles) - t0, SWIGLU ? BN / 32 : BN / 16);
  const uint8_t* wp[2] = {a.wp + (size_t)t0 * KS * 1024, a.wp + (size_t)((SWIGLU ? half : 0) + t0) * KS * 1024};
  const int wbytes = wt * KS * 1024;  // tiles past W read as zero
  i32x4 w[D][TN];
  auto fetch = [&](int own, int d) {
    const int s = KG == 1 ? own : 2 * own + kg;
#pragma unroll
    for (int n = 0; n < TN; ++n) {
      const int x = wn * TN + n, t = SWIGLU ? x >> 1 : x;
      w[d][n] = __builtin_bit_cast(
          i32x4, __builtin_amdgcn_raw_buffer_load_b128(
                     __builtin_amdgcn_make_buffer_rsrc((void*)wp[SWIGLU ? n & 1 : 0], (short)0, s < KS ? wbytes : 0, 0x00020000),
                     (uint32_t)(lane * 16 + (t * KS + s) * 1024), 0, 0));
    }
  };

  i32x4 acc[TN][TM];
#pragma unroll
  for (int n = 0; n < TN; ++n)
#pragma unroll
    for (int m = 0; m < TM; ++m) acc[n][m] = i32x4{0, 0, 0, 0};
  i32x4 fx[LA];
  const int xr = c16 * 128;
  // of the own step p of a slab
  const int xc[2] = {((KG == 1 ? 0 : 4 * kg) + q ^ (c16 >> 1)) * 16, (4 + q ^ (c16 >> 1)) * 16};
  auto wait = [](auto n) {
    constexpr int N = decltype(n)::value;
    __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | 0x0070);  // vmcnt(N), lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
#pragma unroll
  for (int i = 0; i < NX - 1; ++i) issue_x(i, smem + i * XS);
#pragma unroll
  for (int d = 0; d < D; ++d) fetch(d, d);
  wait(std::integral_constant<int, (NX - 2) * PX + D * TN>{});
  char *xs = smem, *xfree = smem + (NX - 1) * XS;  // this slab's stage, and the one before it
#pragma unroll
  for (int i = 0; i < LA; ++i) fx[i] = *(const i32x4*)(xs + xr + xc[0] + i * 2048);
  int slab = 0;
  for (int own = 0; own < KS / KG; own += D) {
#pragma unroll
    for (int d = 0; d < D; ++d) {
      constexpr int LAST = SP - 1;
      const int p = d % SP;
      const char* xnext = xs;
      if (p == LAST) {
        // the next slab of x has landed (behind it came NX - 3 slabs and W of NX - 2 slabs' steps), and the one before
        // this has been read by all
        wait(std::integral_constant<int, (NX - 3) * PX + (D < (NX - 2) * SP ? D : (NX - 2) * SP) * TN>{});
        xnext = xs == smem + (NX - 1) * XS ? smem : xs + XS;
        issue_x(slab + NX - 1, xfree);
      }
#pragma unroll
      for (int m = 0; m < TM; ++m) {
#pragma unroll
        for (int n = 0; n < TN; ++n) {
          acc[n][m] = mfma_i8(w[d][n], fx[m % LA], acc[n][m]);
          __builtin_amdgcn_sched_barrier(0x406);
        }
        const int f = m + LA;
        fx[m % LA] = *(const i32x4*)((f < TM ? xs : xnext) + xr + xc[f < TM ? p : (p + 1) % SP] + f % TM * 2048);
        __builtin_amdgcn_sched_barrier(0x406);
      }
      fetch(own + d + D, d);
      if (p == LAST) {
        xfree = xs;
        xs = (char*)xnext;
        ++slab;
      }
    }
  }
  __builtin_amdgcn_s_waitcnt(0x0070);  // nothing of this workgroup's is on its way into LDS

  if constexpr (KG > 1) {
    __syncthreads();
    i32x4* red = (i32x4*)smem + wn * TM * TN * 64 + lane;
    if (kg == 1) {
#pragma unroll
      for (int n = 0; n < TN; ++n)
#pragma unroll
        for (int m = 0; m < TM; ++m) red[(n * TM + m) * 64] = acc[n][m];
    }
    __syncthreads();
    if (kg == 1) return;
#pragma unroll
    for (int n = 0; n < TN; ++n)
#pragma unroll
      for (int m = 0; m < TM; ++m) acc[n][m] += red[(n * TM + m) * 64];
  }

  const float* sw = (const float*)(a.wp + code_bytes(a.N, a.K));
  const int N = SWIGLU ? a.N / 2 : a.N;
  constexpr int TO = SWIGLU ? TN / 2 : TN;  // tiles of outputs
  const int to = t0 + wn * TO, last = (SWIGLU ? half : ntiles) - 1;
  by_output(a, [&](auto wide, auto f32) {
    const Rows<wide.value, f32.value> io(a, m0, rows, N);
    f32x4 ws[TO], us[SWIGLU ? TO : 1];
#pragma unroll
    for (int n = 0; n < TO; ++n) {
      const int t = min(to + n, last);
      ws[n] = *(const f32x4*)(sw + t * 16 + q * 4);
      if constexpr (SWIGLU) us[n] = *(const f32x4*)(sw + (half + t) * 16 + q * 4);
    }
    // a row at a time: its residuals are all asked for before its results are stored
#pragma unroll
    for (int m = 0; m < TM; ++m) {
      const int row = m * 16 + c16;
      const bool in = row < rows;
      const float sx = a.sx[m0 + min(row, rows - 1)];
      const uint32_t at = row * (uint32_t)a.ldo;
      f32x4 y[TO];
#pragma unroll
      for (int n = 0; n < TO; ++n) {
        const i32x4 v = acc[SWIGLU ? 2 * n : n][m];
#pragma unroll
        for (int x = 0; x < 4; ++x) y[n][x] = (float)v[x] * sx * ws[n][x];
        if constexpr (SWIGLU) {
          const i32x4 u = acc[2 * n + 1][m];
#pragma unroll
          for (int x = 0; x < 4; ++x) y[n][x] = silu_of(y[n][x]) * ((float)u[x] * sx * us[n][x]);
        }
      }
      if (a.res) {
#pragma unroll
        for (int n = 0; n < TO; ++n) {
          const int col = row_of(to + n, 4 * q);
          y[n] += io.residual(at + col, col, in);
        }
      }
#pragma unroll
      for (int n = 0; n < TO; ++n) {
        const int col = row_of(to + n, 4 * q);
        io.store(at + col, col, in, y[n]);
      }
    }
  });
}

template <int BM, int BN, int WGN, int KG, int NX, int D, int LA>
hipError_t launch_tile(const GemmI8Args& a, hipStream_t s) {
  const int64_t wgs = ((int64_t)a.M + BM - 1) / BM * ((a.N + BN - 1) / BN);
  if (wgs >= (1ll << 32) / (64 * WGN * KG)) return hipErrorInvalidValue;  // threads of a launch
  const dim3 grid((unsigned)wgs), block(64 * WGN * KG);
  if (a.swiglu) {
    if constexpr (BN / WGN % 32 == 0)
      hipLaunchKernelGGL((w8_tile_kernel<BM, BN, WGN, KG, NX, D, LA, true>), grid, block, 0, s, a);
    else
      return hipErrorInvalidValue;
  } else {
    hipLaunchKernelGGL((w8_tile_kernel<BM, BN, WGN, KG, NX, D, LA, false>), grid, block, 0, s, a);
  }
  return hipGetLastError();
}
template <int NT, int W, int U>
hipError_t launch_rows(const GemmI8Args& a, hipStream_t s) {
  const dim3 grid(cdiv(a.swiglu ? tiles_of(a.N) / 2 : tiles_of(a.N), a.swiglu ? NT / 2 : NT)), block(W * 64);
  if constexpr (NT > 1) {
    if (a.swiglu) {
      hipLaunchKernelGGL((w8_rows_kernel<NT, W, U, true>), grid, block, 0, s, a);
      return hipGetLastError();
    }
  }
  hipLaunchKernelGGL((w8_rows_kernel<NT, W, U, false>), grid, block, 0, s, a);
  return hipGetLastError();
}

// The tile of a product over more than 16 rows: the one whose estimated time is least.
// Workgroups run in rounds of 256 per_cu; a workgroup takes t us for a slab of 128 k and f us
// for its ends, and t grows with the number that run together, since they share L2 and,
// past 256, a CU: t0 for few, t1 for one on every CU, step more as the first CUs take a
// second one, t2 for two on every CU, t3 for three.  The figures are a least-squares fit to 7000
// products timed in every tile with their weights read from memory (M = 17 to 4096, N =
// 256 to 22016, K = 256 to 11008; mean error 9 to 13%); what the choice takes is
// 1.8% slower than the fastest tile on average, 23% in one of a hundred, 39% at most.  us,
// the same products in each tile:
//                                        128x512 128x256 64x256 128x128 64x128 48x128 64x64 32x64 32x32
//   2048 x 22016, K =  4096, gated            160     161    206     185    242    252   273   407   464 (from cache)
//   2048 x 12288, K =  4096                   107      92    128     111    149    153   165   236   268
//    333 x  4096, K = 11008, residual         121      72     58      51     37     37    43    50    62
//    333 x  4096, K = 11008, residual          98      55     40      39     29     26    33    38    52 (from cache)
//     64 x  4096, K = 11008, residual          93      51     40      32     27     24    20    16    14 (from cache)
struct Tile {
  int rows, cols, per_cu;
  float t0, t1, step, t2, t3, f;
};
constexpr Tile kTiles[] = {
    {128, 512, 1, 0.984f, 1.819f, 0.f, 0.f, 0.f, 9.08f},        {128, 256, 1, 0.546f, 0.950f, 0.f, 0.f, 0.f, 5.49f},
    {64, 256, 2, 0.390f, 0.767f, 0.432f, 1.276f, 0.f, 3.61f},   {128, 128, 2, 0.335f, 0.689f, 0.432f, 1.130f, 0.f, 5.90f},
    {64, 128, 2, 0.248f, 0.461f, 0.351f, 0.728f, 0.f, 3.83f},   {48, 128, 2, 0.216f, 0.440f, 0.344f, 0.673f, 0.f, 3.25f},
    {64, 64, 3, 0.158f, 0.270f, 0.135f, 0.660f, 0.674f, 3.54f}, {32, 64, 3, 0.115f, 0.197f, 0.125f, 0.480f, 0.465f, 2.48f},
    {32, 32, 3, 0.079f, 0.115f, 0.074f, 0.338f, 0.278f, 2.67f}};
constexpr int kTileCount = sizeof(kTiles) / sizeof(kTiles[0]);
int choose_tile(int M, int N, int K) {
  const float slabs = (float)(steps_of(K) / 2);
  int best = 0;
  float least = 0.f;
  for (int i = 0; i < kTileCount; ++i) {
    const Tile& t = kTiles[i];
    const int64_t wgs = ((int64_t)M + t.rows - 1) / t.rows * (((int64_t)N + t.cols - 1) / t.cols), round = 256 * t.per_cu;
    auto slab_us = [&](int64_t n) {
      const float x = (float)n / 256.f;
      return x <= 1.f   ? t.t0 + (t.t1 - t.t0) * x
             : x <= 2.f ? t.t1 + t.step + (t.t2 - t.t1 - t.step) * (x - 1.f)
                        : t.t2 + (t.t3 - t.t2) * (x - 2.f);
    };
    float us = (float)(wgs / round) * (slab_us(round) * slabs + t.f);
    if (wgs % round) us += slab_us(wgs % round) * slabs + t.f;
    if (i == 0 || us < least) least = us, best = i;
  }
  return best;
}

// One thread per 16 bytes of the packed codes, then the scales.
__global__ __launch_bounds__(256) void w8_pack_kernel(const int8_t* __restrict__ codes, const float* __restrict__ scales,
                                                      uint8_t* __restrict__ wp, int N, int K) {
  const int KS = steps_of(K);
  const size_t nc = code_bytes(N, K) / 16, ns = (size_t)tiles_of(N) * 16;
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < nc + ns; i += (size_t)gridDim.x * 256) {
    if (i < nc) {
      const int lane = (int)(i & 63);
      const size_t blk = i >> 6;
      const int n = row_of((int)(blk / KS), lane & 15), k = (int)(blk % KS) * 64 + (lane >> 4) * 16;
      u32x4 v = {0u, 0u, 0u, 0u};
      if (n < N && k < K) v = *(const u32x4*)(codes + (size_t)n * K + k);  // K % 16 == 0
      *(u32x4*)(wp + i * 16) = v;
    } else {
      const int r = (int)(i - nc), n = row_of(r >> 4, r & 15);
      ((float*)(wp + nc * 16))[r] = n < N ? scales[n] : 0.f;
    }
  }
}

}  // namespace

size_t w8_packed_bytes(int N, int K) { return code_bytes(N, K) + (size_t)tiles_of(N) * 64; }

hipError_t w8_pack(const int8_t* codes, const float* scales, void* wp, int N, int K, hipStream_t s) {
  const size_t n = code_bytes(N, K) / 16 + (size_t)tiles_of(N) * 16;
  const unsigned grid = (unsigned)((n + 255) / 256 < 65536 ? (n + 255) / 256 : 65536);
  hipLaunchKernelGGL(w8_pack_kernel, dim3(grid), dim3(256), 0, s, codes, scales, (uint8_t*)wp, N, K);
  return hipGetLastError();
}

void gemm_i8_tile(int M, int N, int K, int* rows, int* cols) {
  const Tile t = M > 16 ? kTiles[choose_tile(M, N, K)] : Tile{};
  *rows = t.rows;
  *cols = t.cols;
}

hipError_t gemm_i8(const GemmI8Args& a, hipStream_t s) {
  if (a.M <= 16) {
    // waves and tiles a workgroup by the number of tiles.  us, weights from memory, of one row (of 16): 8 waves, 4 waves, 8
    // waves of two tiles
    //    2048, K = 2048   3.0  3.5  3.6 ( 3.6  4.1  4.2)      12288, K = 4096  11.4 11.4 12.1 (14.2 13.9 13.4)
    //    4096, K = 4096   5.8  6.5  6.3 ( 6.6  7.2  7.6)      16416, K = 4096  15.1 14.7 15.5 (19.3 19.7 17.7)
    //    8192, K = 4096   8.6  8.4  8.4 (10.0 10.3  9.1)      22016, K = 4096  18.6 18.4 17.7 (25.0 25.5 20.1)
    //    8224, K = 4096  10.0  9.8 10.6 (12.6 12.6 12.2)      57344, K = 8192  78   79   77   ( 111  112   86)
    // What lies between is flat for one row; with 16 two tiles are faster from N = 6144 on.
    if (a.swiglu) return launch_rows<2, 8, 2>(a, s);
    return a.N <= 8192    ? launch_rows<1, 8, 4>(a, s)
           : a.N <= 16384 ? launch_rows<1, 4, 4>(a, s)
                          : launch_rows<2, 8, 2>(a, s);
  }
  switch (choose_tile(a.M, a.N, a.K)) {  // the table's order
    case 0: return launch_tile<128, 512, 8, 1, 3, 4, 4>(a, s);
    case 1: return launch_tile<128, 256, 8, 1, 4, 4, 4>(a, s);
    case 2: return launch_tile<64, 256, 8, 1, 4, 4, 4>(a, s);
    case 3: return launch_tile<128, 128, 4, 2, 4, 4, 4>(a, s);
    case 4: return launch_tile<64, 128, 4, 2, 4, 4, 4>(a, s);
    case 5: return launch_tile<48, 128, 4, 2, 6, 4, 3>(a, s);
    case 6: return launch_tile<64, 64, 2, 2, 6, 4, 4>(a, s);
    case 7: return launch_tile<32, 64, 2, 2, 6, 4, 2>(a, s);
    default: return launch_tile<32, 32, 1, 2, 8, 8, 2>(a, s);
  }
}

}  // namespace vla
