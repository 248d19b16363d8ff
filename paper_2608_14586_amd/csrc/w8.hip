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
// Up to 16 MT rows of x: the weights' bytes are the bound.  A workgroup takes NT
// tiles of weight rows (SWIGLU: NT / 2 gate tiles and the up tiles of the same
// features); its W waves take runs of U steps in turn and add up in LDS.  Weights go
// from memory into registers, a run ahead.
template <int NT, int MT, int W, int U, bool SWIGLU>
__global__ __launch_bounds__(W * 64) void w8_rows_kernel(GemmI8Args a) {
  __shared__ i32x4 part[W][NT * MT][64];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c16 = lane & 15, q = lane >> 4;
  const int KS = steps_of(a.K), ntiles = tiles_of(a.N), half = ntiles / 2;
  constexpr int TW = SWIGLU ? NT / 2 : NT;
  const int t0 = blockIdx.x * TW, m0 = blockIdx.y * (16 * MT);
  const int rows = min(a.M - m0, 16 * MT);
  const uint8_t* wt[NT];
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    const int t = SWIGLU ? (i < TW ? min(t0 + i, half - 1) : half + min(t0 + i - TW, half - 1)) : min(t0 + i, ntiles - 1);
    wt[i] = a.wp + (size_t)t * KS * 1024;
  }
  // past the row of x: its next one, or zeros past the last; the weights there are zero
  const uint8_t* xp = (const uint8_t*)a.x + (int64_t)m0 * a.ldx;
  const uint32_t xbytes = (uint32_t)((rows - 1) * a.ldx + a.K);
  uint32_t xat[MT];
#pragma unroll
  for (int j = 0; j < MT; ++j) {
    const int r = j * 16 + c16;
    xat[j] = r < rows ? (uint32_t)(r * a.ldx) + q * 16 : 0x80000000u;
  }
  i32x4 wr[2][NT][U], xr[2][MT][U];
  auto fetch = [&](int b, int s0) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool in = s0 + u < KS;
#pragma unroll
      for (int i = 0; i < NT; ++i)
        wr[b][i][u] = __builtin_bit_cast(
            i32x4, __builtin_amdgcn_raw_buffer_load_b128(
                       __builtin_amdgcn_make_buffer_rsrc((void*)wt[i], (short)0, in ? KS * 1024 : 0, 0x00020000),
                       lane * 16, in ? (s0 + u) * 1024 : 0, 0));
#pragma unroll
      for (int j = 0; j < MT; ++j)
        xr[b][j][u] = __builtin_bit_cast(
            i32x4, __builtin_amdgcn_raw_buffer_load_b128(
                       __builtin_amdgcn_make_buffer_rsrc((void*)xp, (short)0, in ? (int)xbytes : 0, 0x00020000), xat[j],
                       in ? (s0 + u) * 64 : 0, 0));
    }
  };
  i32x4 acc[NT][MT];
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int j = 0; j < MT; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
  auto multiply = [&](int b) {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int j = 0; j < MT; ++j) acc[i][j] = mfma_i8(wr[b][i][u], xr[b][j][u], acc[i][j]);
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
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int j = 0; j < MT; ++j) part[wave][i * MT + j][lane] = acc[i][j];
  __syncthreads();
  const float* sw = (const float*)(a.wp + code_bytes(a.N, a.K));
  const int N = SWIGLU ? a.N / 2 : a.N;
  for (int e = wave; e < TW * MT; e += W) {
    const int i = e / MT, j = e % MT;
    const int m = j * 16 + c16, t = min(t0 + i, (SWIGLU ? half : ntiles) - 1), col = row_of(t0 + i, 4 * q);
    auto joined = [&](int i) {
      i32x4 v = part[0][i * MT + j][lane];
#pragma unroll
      for (int w = 1; w < W; ++w) v += part[w][i * MT + j][lane];
      return v;
    };
    const i32x4 v = joined(i), g = SWIGLU ? joined(i + TW) : v;
    const float sx = a.sx[m0 + min(m, rows - 1)];
    const f32x4 ws = *(const f32x4*)(sw + t * 16 + q * 4);  
    f32x4 y;
#pragma unroll
    for (int x = 0; x < 4; ++x) y[x] = (float)v[x] * sx * ws[x];
    if constexpr (SWIGLU) {
      const f32x4 us = *(const f32x4*)(sw + (half + t) * 16 + q * 4);
#pragma unroll
      for (int x = 0; x < 4; ++x) y[x] = silu_of(y[x]) * ((float)g[x] * sx * us[x]);
    }
    by_output(a, [&](auto wide, auto f32) {
      const Rows<wide.value, f32.value> io(a, m0, rows, N);
      const uint32_t at = m * (uint32_t)a.ldo + col;
      if (a.res) y += io.residual(at, col, m < rows);
      io.store(at, col, m < rows, y);
    });
  }
}

// ----------------------------------------------------------------- many rows
//
// A workgroup of 64 NW threads takes BM rows of x by BN rows of W.  Slabs of KG
// steps of 64 k move to LDS by buffer_load ... lds in a ring of NS stages, both
// operands in MFMA order (1024 bytes a tile and step, lane l's operand at 16 l), so
// that every read of an operand is 64 lanes side by side, free of bank conflicts
// without a swizzle.  While the MFMAs of slab i run, its successor's operands are
// read into registers and slab i + NS is on its way into the stage that slab i left.
// KG = 2: half of the waves take the even steps, half the odd ones, and add up in LDS.
template <int BM, int BN, int WGM, int WGN, int KG, int NS, bool SWIGLU>
__global__ __launch_bounds__(64 * WGM * WGN * KG) void w8_tile_kernel(GemmI8Args a) {
  constexpr int NW = WGM * WGN * KG, WM = BM / WGM, WN = BN / WGN, TM = WM / 16, TN = WN / 16;
  constexpr int AB = BM / 16 * KG, WB = BN / 16 * KG, PA = AB / NW, PW = WB / NW, PER = PA + PW;  // 1 KB blocks
  constexpr int STAGE = (AB + WB) * 1024;
  static_assert(PA * NW == AB && PW * NW == WB, "blocks divide over the waves");
  static_assert((NS - 2) * PER < 64, "vmcnt range");
  static_assert(!SWIGLU || WN % 64 == 0, "a wave's tiles must be whole (gate, up) groups");
  constexpr int RED = KG > 1 ? WGM * WGN * TM * TN * 1024 : 0;
  __shared__ __attribute__((aligned(1024))) char smem[NS * STAGE > RED ? NS * STAGE : RED];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kg = wave / (WGM * WGN), wm = wave / WGN % WGM, wn = wave % WGN;
  const int c16 = lane & 15, q = lane >> 4;
  const int KS = steps_of(a.K), ntiles = tiles_of(a.N), half = ntiles / 2;
  const int nslab = KS / KG;

  // tiles: each of the 8 XCDs takes a contiguous run of them, walked M first inside
  // groups of 8 tile rows
  const int tiles_m = (a.M + BM - 1) / BM, tiles_n = (a.N + BN - 1) / BN;
  const int nwg = gridDim.x;
  int id = blockIdx.x;
  {
    const int per = nwg >> 3, rem = nwg & 7, x = id & 7;
    id = x * per + min(x, rem) + (id >> 3);
  }
  const int group = 8 * tiles_n, first_m = id / group * 8, gsz = min(tiles_m - first_m, 8);
  const int m0 = (first_m + id % group % gsz) * BM, tile_n = id % group / gsz;
  const int t0 = SWIGLU ? tile_n * (BN / 32) : tile_n * (BN / 16);  // first tile of W (of the gate's)

  const int rows = min(a.M - m0, BM);
  const uint8_t* xp = (const uint8_t*)a.x + (int64_t)m0 * a.ldx;
  const int xbytes = (int)((rows - 1) * a.ldx + a.K);
  const uint8_t* wp0 = a.wp + (size_t)t0 * KS * 1024;
  const uint8_t* wp1 = SWIGLU ? a.wp + (size_t)(half + t0) * KS * 1024 : wp0;
  const int wt = min((SWIGLU ? half : ntiles) - t0, SWIGLU ? BN / 32 : BN / 16);
  const int wbytes = wt * KS * 1024;

  // this wave's blocks of a slab: x block j is tile (wave PA + j) / KG, step (wave PA + j) % KG
  const uint32_t xvoff = (uint32_t)(c16 * a.ldx) + q * 16, wvoff = lane * 16;
  auto issue = [&](int slab, char* st) {
    const bool in = slab < nslab;  // past the last: empty buffers, no memory touched
    const __amdgpu_buffer_rsrc_t rx = __builtin_amdgcn_make_buffer_rsrc((void*)xp, (short)0, in ? xbytes : 0, 0x00020000);
#pragma unroll
    for (int j = 0; j < PA; ++j) {
      const int blk = wave * PA + j, t = blk / KG, s = blk % KG;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rx, (__attribute__((address_space(3))) void*)(st + blk * 1024), 16, xvoff,
                                               (int)(t * 16 * a.ldx) + (slab * KG + s) * 64, 0, 0);
    }
#pragma unroll
    for (int j = 0; j < PW; ++j) {
      const int blk = wave * PW + j, t = blk / KG, s = blk % KG;
      // SWIGLU: two gate tiles, then the two up tiles of the same features
      const bool up = SWIGLU && (t & 2);
      const int tt = SWIGLU ? (t >> 2) * 2 + (t & 1) : t;
      const __amdgpu_buffer_rsrc_t rw = __builtin_amdgcn_make_buffer_rsrc((void*)(up ? wp1 : wp0), (short)0, in ? wbytes : 0, 0x00020000);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rw, (__attribute__((address_space(3))) void*)(st + (AB + blk) * 1024), 16,
                                               wvoff, (tt * KS + slab * KG + s) * 1024, 0, 0);
    }
  };

  i32x4 acc[TN][TM];
#pragma unroll
  for (int n = 0; n < TN; ++n)
#pragma unroll
    for (int m = 0; m < TM; ++m) acc[n][m] = i32x4{0, 0, 0, 0};
  i32x4 fx[2][TM], fw[2][TN];
  const int xread = (wm * TM * KG + kg) * 1024 + lane * 16, wread = (AB + wn * TN * KG + kg) * 1024 + lane * 16;
  auto read = [&](const char* st, int i, int b) {
    if (i < TN)
      fw[b][i] = *(const i32x4*)(st + wread + i * KG * 1024);
    else
      fx[b][i - TN] = *(const i32x4*)(st + xread + (i - TN) * KG * 1024);
  };
  auto wait = [](auto n) {
    constexpr int N = decltype(n)::value;
    __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | 0x0070);  // vmcnt(N), lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
#pragma unroll
  for (int i = 0; i < NS; ++i) issue(i, smem + i * STAGE);
  wait(std::integral_constant<int, (NS - 1) * PER>{});
#pragma unroll
  for (int i = 0; i < TM + TN; ++i) read(smem, i, 0);

  // the stages of slab i and of slab i + 1 (an even number of slabs in all)
  char *st = smem, *next = smem + STAGE;
  for (int base = 0; base < nslab; base += 2) {
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      // slab i + 1 has landed for every wave, and every wave has read slab i
      wait(std::integral_constant<int, (NS - 2) * PER>{});
      issue(base + b + NS, st);
      constexpr int NMF = TM * TN, NR = TM + TN, EVERY = NMF / NR > 0 ? NMF / NR : 1;
      int r = 0;
#pragma unroll
      for (int x = 0; x < NMF; ++x) {
        if (x % EVERY == 0 && r < NR) read(next, r++, b ^ 1);
        const int n = x / TM, m = x % TM;
        acc[n][m] = mfma_i8(fw[b][n], fx[b][m], acc[n][m]);
        __builtin_amdgcn_sched_barrier(0x406);
      }
#pragma unroll
      for (; r < NR; ++r) read(next, r, b ^ 1);
      st = next;
      next = next == smem + (NS - 1) * STAGE ? smem : next + STAGE;
    }
  }
  __builtin_amdgcn_s_waitcnt(0x0070);  // nothing of this workgroup's on its way into LDS

  if constexpr (KG > 1) {
    __syncthreads();
    i32x4* red = (i32x4*)smem + (wm * WGN + wn) * TM * TN * 64 + lane;
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
      const int row = wm * WM + m * 16 + c16;
      const bool in = row < rows;
      const float sx = a.sx[m0 + min(row, rows - 1)];
      const uint32_t at = row * (uint32_t)a.ldo;
      f32x4 y[TO];
#pragma unroll
      for (int n = 0; n < TO; ++n) {
        const i32x4 v = acc[SWIGLU ? n / 2 * 4 + n % 2 : n][m];
#pragma unroll
        for (int x = 0; x < 4; ++x) y[n][x] = (float)v[x] * sx * ws[n][x];
        if constexpr (SWIGLU) {
          const i32x4 u = acc[n / 2 * 4 + 2 + n % 2][m];
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

template <int BM, int BN, int WGM, int WGN, int KG, int NS>
hipError_t launch_tile(const GemmI8Args& a, hipStream_t s) {
  const int64_t wgs = ((int64_t)a.M + BM - 1) / BM * ((a.N + BN - 1) / BN);
  if (wgs >= (1ll << 32) / (64 * WGM * WGN * KG)) return hipErrorInvalidValue;  // threads of a launch
  const dim3 grid((unsigned)wgs), block(64 * WGM * WGN * KG);
  if (a.swiglu)
    hipLaunchKernelGGL((w8_tile_kernel<BM, BN, WGM, WGN, KG, NS, true>), grid, block, 0, s, a);
  else
    hipLaunchKernelGGL((w8_tile_kernel<BM, BN, WGM, WGN, KG, NS, false>), grid, block, 0, s, a);
  return hipGetLastError();
}
template <int NT, int MT, int W, int U>
hipError_t launch_rows(const GemmI8Args& a, hipStream_t s) {
  const int tiles = a.swiglu ? tiles_of(a.N) / 2 : (a.N + 15) / 16, tw = a.swiglu ? NT / 2 : NT;
  const dim3 grid(cdiv(tiles, tw), cdiv(a.M, 16 * MT)), block(W * 64);
  if constexpr (NT > 1) {
    if (a.swiglu) {
      hipLaunchKernelGGL((w8_rows_kernel<NT, MT, W, U, true>), grid, block, 0, s, a);
      return hipGetLastError();
    }
  }
  hipLaunchKernelGGL((w8_rows_kernel<NT, MT, W, U, false>), grid, block, 0, s, a);
  return hipGetLastError();
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

hipError_t gemm_i8(const GemmI8Args& a, hipStream_t s) {
  if (a.M <= 16) return launch_rows<2, 1, 8, 4>(a, s);
  if ((int64_t)a.M * a.N >= 256ll * 256 * 200) return launch_tile<256, 256, 2, 4, 1, 4>(a, s);
  return launch_tile<128, 128, 2, 2, 1, 4>(a, s);
}

}  // namespace vla
