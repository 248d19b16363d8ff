// The KV cache in 8 bits: rows into it, rows out of it, and attention over it.
//
// A block is 32 positions of one sequence and KV head.  Its keys share a power of two
// 2^e, its values another; a number is held as c 2^e, c a float of 8 bits (4 of
// exponent, 3 of mantissa, at most 448).  A power of two, because then a block whose exponent
// grows with a new row keeps its codes but for the smallest: c is divided by a power of
// two, exactly where it does not reach the 2^-9 steps of the smallest codes.
//
// The cache is the codes of all blocks, sequence by sequence, head by head, 64 dh
// bytes each, then two fp32 steps 2^e a block (keys, values).  A block is
//   key codes    [tile 2][dh / 64][lane 64][2][8]: lane l's 8 codes of token 16 tile +
//                l % 16, dims 64 i + 32 j + 8 (l / 16) ..
//   value codes  [dh / 32][lane 64][2][8]: lane l's codes of dim 32 i + 16 j + l % 16,
//                tokens 4 (l / 16) .. + 3 and 16 + 4 (l / 16) .. + 3
// so that a wave's loads are contiguous, 16 bytes a lane, and every 8 codes are a lane's
// operand of one MFMA step.
#include <limits.h>

#include <type_traits>

#include "kernels.h"

namespace vla {
namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr int BLK = 32;        // positions per block
constexpr int LEAST_E = -118;  // of a block's exponent: codes' smallest steps are then fp32's too

// ------------------------------------------------------------ rows in and out

// this workgroup's block of the cache and the tokens of the call in it: positions
// [t0, t1) of the block are tokens from + (t - t0) of the sequence's rows
struct Span {
  int b, h, blk, t0, t1, from;
};
__device__ __forceinline__ Span span_of(const Kv8Rows& a, int wg) {
  Span s;
  // the heads of a block side by side: so are their rows of a token, where heads are inner
  const int bi = div_by(wg, a.by_Hkv);
  s.h = wg - bi * a.Hkv;
  s.b = div_by(bi, a.by_blocks);
  const int i = bi - s.b * a.blocks;
  const int64_t start = a.start ? a.start[s.b] : 0;
  const int count = a.count ? min(max(a.count[s.b], 0), a.L) : a.L;
  // rows [first, last) of the cache, cut to the rows that it has
  const int64_t first = max(start, (int64_t)0), last = min(start + count, (int64_t)a.L_cap);
  const int64_t blk = first / BLK + i;
  const int64_t lo = max(first, blk * BLK), hi = min(last, (blk + 1) * BLK);
  s.blk = (int)blk;
  s.t0 = (int)(lo - blk * BLK);
  s.t1 = hi > lo ? (int)(hi - blk * BLK) : s.t0;
  s.from = (int)(lo - start);
  return s;
}

// the exponent that a block with the largest magnitude `mag` (a finite bf16's bits) needs:
// 448 is 1.75 2^8
__device__ __forceinline__ int exponent_for(uint32_t mag) {
  return max((int)(mag >> 7) - 127 - 8 + ((mag & 0x7f) > 0x60 ? 1 : 0), LEAST_E);
}
__device__ __forceinline__ float power2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}
// four codes times f, rounded to codes again
__device__ __forceinline__ uint32_t rescale4(uint32_t w, float f) {
  const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  uint32_t r = codes4(a[0] * f, a[1] * f, b[0] * f, b[1] * f);
  // NaN stays as it is
  const uint32_t nan = (((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) >> 7;
  const uint32_t all = nan * 255u;
  return (r & ~all) | (w & all);
}

// One workgroup for the keys of a block (even ones) or for its values.  Every thread
// quantises a piece of a row, the codes cross LDS, and every thread writes 16 bytes of
// the block as it lies in memory, with the codes of positions that the call does not
// store as they were (or rescaled, where the block's exponent grows).  Memory bounds it:
// 2048 tokens of 32 heads of 128, 50 MB in all, take 13.1 us (3.8 TB/s, the launch's 2.3 us
// included), a token of each of four sequences of two heads 3.3.  Values transposed in
// registers and all rows in whole cache lines through LDS measured 13.2 us, keys and values
// in one workgroup 13.7 and 3.9.  Sequences that share all rows have a workgroup for each block that any of
// them might touch: 12 prompts in 8192 rows, 32 heads of 128, 104 us where one sequence of 8192 takes 42, 64
// prompts, 8 heads, 109 for 12.
template <int DH>
__global__ __launch_bounds__(2 * DH) void kv8_store_kernel(Kv8Rows a) {
  constexpr int T = 2 * DH, W = T / 64, TPR = T / BLK, V = DH / TPR;  // threads a row, values a thread: 16
  static_assert(V == 16, "two pieces of 8 a thread");
  constexpr int ROWB = DH + 4;
  __shared__ __attribute__((aligned(16))) uint8_t cs[BLK * ROWB];
  __shared__ uint32_t tops[W];
  const Span s = span_of(a, blockIdx.x >> 1);
  const int values = blockIdx.x & 1;
  if (s.t0 >= s.t1) return;
  const size_t block = ((size_t)s.b * a.Hkv + s.h) * (a.L_cap / BLK) + s.blk;
  u32x4* image = (u32x4*)((uint8_t*)a.cache + block * (64 * DH) + values * (32 * DH));
  float* step = (float*)((uint8_t*)a.cache + (size_t)a.B * a.Hkv * (a.L_cap / BLK) * (64 * DH)) + block * 2 + values;
  const int tid = threadIdx.x;
  const int t = tid / TPR, d0 = tid % TPR * V;
  const bool there = t >= s.t0 && t < s.t1;
  const bool anew = s.t0 == 0;
  const Heads& in = values ? a.v : a.k;
  u32x4 x[2] = {{0u, 0u, 0u, 0u}, {0u, 0u, 0u, 0u}};
  if (there) {
    const u32x4* row = (const u32x4*)((const bf16_t*)in.p + s.b * in.seq + (int64_t)(s.from + t - s.t0) * in.token + s.h * in.head + d0);
    x[0] = row[0];
    x[1] = row[1];
  }
  u32x4 old = {0u, 0u, 0u, 0u};
  float was = 0.f;
  if (!anew) {
    old = image[tid];
    was = *step;
  }
  // the largest finite magnitude, as whole numbers
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t lo = x[i][e] & 0x7fffu, hi = x[i][e] >> 16 & 0x7fffu;
      top = max(top, max(lo < 0x7f80u ? lo : 0u, hi < 0x7f80u ? hi : 0u));
    }
  top = wave_max_u(top);
  if (tid % 64 == 0) tops[tid / 64] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < W; ++w) top = max(top, tops[w]);
  const float need = power2(exponent_for(top)), now = anew ? need : fmaxf(was, need);
  const float inv = __uint_as_float(0x7f000000u - __float_as_uint(now));  // 1 / now
  if (there) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float f[8];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        f[2 * e] = __uint_as_float(x[i][e] << 16);
        f[2 * e + 1] = __uint_as_float(x[i][e] & 0xffff0000u);
      }
      uint32_t w[2], bad = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) bad |= (__float_as_uint(f[e]) & 0x7fffffffu) >= 0x7f800000u ? 1u << e : 0u;
      w[0] = codes4(f[0] * inv, f[1] * inv, f[2] * inv, f[3] * inv);
      w[1] = codes4(f[4] * inv, f[5] * inv, f[6] * inv, f[7] * inv);
      if (bad)
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (bad >> e & 1) w[e / 4] |= 0x7fu << e % 4 * 8;
      uint32_t* to = (uint32_t*)(cs + t * ROWB + d0 + i * 8);
      to[0] = w[0];
      to[1] = w[1];
    }
  }
  __syncthreads();
  // 16 bytes of the block, and which of them are of stored positions
  const int lane = tid & 63, c = lane & 15, q = lane >> 4, piece = tid >> 6;
  u32x4 w, mine;
  if (!values) {
    const int tt = piece / (DH / 64) * 16 + c, d = piece % (DH / 64) * 64 + q * 8;
    const uint32_t* row = (const uint32_t*)(cs + tt * ROWB + d);
    w = u32x4{row[0], row[1], row[8], row[9]};
    const uint32_t m = tt >= s.t0 && tt < s.t1 ? 0xffffffffu : 0u;
    mine = u32x4{m, m, m, m};
  } else {
    uint32_t m[2] = {0u, 0u};
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int tt = h * 16 + q * 4 + r;
        m[h] |= tt >= s.t0 && tt < s.t1 ? 255u << 8 * r : 0u;
      }
    mine = u32x4{m[0], m[1], m[0], m[1]};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t v = 0;
#pragma unroll
      for (int r = 0; r < 4; ++r)
        v |= (uint32_t)cs[((i & 1) * 16 + q * 4 + r) * ROWB + piece * 32 + (i >> 1) * 16 + c] << 8 * r;
      w[i] = v;
    }
  }
  if (!anew && now != was) {  // a power of two, 2^-238 at least; below 2^-126 nothing is left of a code
    const float f = was * inv;
#pragma unroll
    for (int i = 0; i < 4; ++i) old[i] = rescale4(old[i], f);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = (w[i] & mine[i]) | (old[i] & ~mine[i]);
  image[tid] = w;
  if (tid == 0) *step = now;
}

// A block lies in memory as 16 bytes for each thread, of keys those of token 16 t + lane % 16, dims d .. d + 7 and
// d + 32 .. d + 39.  For rows written in whole cache lines they cross LDS: thread tid's part
// of the keys is dims d .. d + 7 of token t and of token t + 16, two words of four codes each.  The pieces of 64 lanes
// lie 16 bytes further apart than in memory, so that the words of a row meet every bank alike.
template <int DH>
struct KeyPart {
  int t, d;
  __device__ __forceinline__ KeyPart(int tid) : t(tid / (DH / 8)), d(tid % (DH / 8) * 8) {}
  // of token t + 16 h
  __device__ __forceinline__ int at(int h) const {
    return ((h * (DH / 64) + d / 64) * 65 + d % 32 / 8 * 16 + t) * 4 + d % 64 / 32 * 2;
  }
};
// And of the values: dims d .. d + 3 of tokens t .. t + 3, four words of four codes.
template <int DH>
struct ValuePart {
  int t, d;
  __device__ __forceinline__ ValuePart(int tid) : t(tid / (DH / 4) * 4), d(tid % (DH / 4) * 4) {}
  // word of dim d + e
  __device__ __forceinline__ int at(int e) const {
    return (d / 32 * 65 + (t / 4 & 3) * 16 + d % 16 + e) * 4 + d % 32 / 16 * 2 + t / 16;
  }
  static constexpr int WORDS = DH / 32 * 65 * 4;
  __device__ static int own(int tid) { return ((tid >> 6) * 65 + (tid & 63)) * 4; }  // of thread tid's 16 bytes
};
// 4 x 4 bytes: byte c of word r becomes byte r of word c
__device__ __forceinline__ void transpose4(uint32_t (&w)[4]) {
  const uint32_t a = __builtin_amdgcn_perm(w[1], w[0], 0x05010400u), b = __builtin_amdgcn_perm(w[1], w[0], 0x07030602u);
  const uint32_t c = __builtin_amdgcn_perm(w[3], w[2], 0x05010400u), d = __builtin_amdgcn_perm(w[3], w[2], 0x07030602u);
  w[0] = __builtin_amdgcn_perm(c, a, 0x05040100u);
  w[1] = __builtin_amdgcn_perm(c, a, 0x07060302u);
  w[2] = __builtin_amdgcn_perm(d, b, 0x05040100u);
  w[3] = __builtin_amdgcn_perm(d, b, 0x07060302u);
}

// The inverse: 16 bytes a thread from memory as they lie, across LDS in words into rows.
// The 50 MB take 10.0 us (5.0 TB/s with the launch), with values picked from LDS byte by byte
// and keys written in half cache lines 10.3.
template <int DH>
__global__ __launch_bounds__(2 * DH) void kv8_load_kernel(Kv8Rows a) {
  __shared__ __attribute__((aligned(16))) uint32_t vs[ValuePart<DH>::WORDS];
  const Span s = span_of(a, blockIdx.x >> 1);
  const bool values = blockIdx.x & 1;
  if (s.t0 >= s.t1) return;
  const size_t block = ((size_t)s.b * a.Hkv + s.h) * (a.L_cap / BLK) + s.blk;
  const u32x4* image = (const u32x4*)((const uint8_t*)a.cache + block * (64 * DH) + values * (32 * DH));
  const float step = ((const float*)((const uint8_t*)a.cache + (size_t)a.B * a.Hkv * (a.L_cap / BLK) * (64 * DH)))[block * 2 + values];
  const int tid = threadIdx.x;
  const u32x4 own = image[tid];
  const Heads& out = values ? a.v : a.k;
  // four codes as bf16: exact, the codes have 4 bits and a power of two keeps them (256 2^120 alone is infinite)
  auto wide = [&](uint32_t w) {
    const f32x2 p = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), q = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    return u32x2{pack_bf2(p[0] * step, p[1] * step), pack_bf2(q[0] * step, q[1] * step)};
  };
  bf16_t* rows = (bf16_t*)out.p + s.b * out.seq + s.h * out.head;
  *(u32x4*)&vs[ValuePart<DH>::own(tid)] = own;
  __syncthreads();
  if (!values) {
    const KeyPart<DH> kp(tid);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int t = kp.t + 16 * h;
      if (t < s.t0 || t >= s.t1) continue;
      const u32x2 lo = wide(vs[kp.at(h)]), hi = wide(vs[kp.at(h) + 1]);
      *(u32x4*)(rows + (int64_t)(s.from + t - s.t0) * out.token + kp.d) = u32x4{lo[0], lo[1], hi[0], hi[1]};
    }
    return;
  }
  const ValuePart<DH> vp(tid);
  uint32_t c[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) c[e] = vs[vp.at(e)];
  transpose4(c);
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int t = vp.t + r;
    if (t >= s.t0 && t < s.t1) *(u32x2*)(rows + (int64_t)(s.from + t - s.t0) * out.token + vp.d) = wide(c[r]);
  }
}

// -------------------------------------------------------------- attention
//
// A decode step's attention reads each visible key and value once for the few queries
// that share its KV head: bound by the cache's bytes.  One wave takes 32 keys at a time:
//  * scores transposed, S^T = K Q^T (16x16x32 bf16 MFMA, key codes as bf16, exact), so
//    that a lane holds 8 keys of one query; the block's step and 1 / sqrt(dh) are one
//    factor a block;
//  * softmax: a running maximum and sum a query in fp32, one pass.  The maximum moves only
//    where a score is 15 (in log2) above it, to 7 below the score: weights lie below 2^15 and are
//    rounded to fp16, off by 2^-11 of each at most (below fp16's normal range by 2^-32 of the largest), an eighth of
//    what the bf16 result's own rounding may be;
//  * O^T = V^T P^T by fp16 MFMA: a lane's 8 weights are the operand as they lie, value
//    codes are fp16 numbers exactly; the block's step is a factor of the block's sum, in
//    fp32, so that no block's step limits another's.  It comes in as 2^-28 of itself:
//    sums of values near the largest bf16 stay in range, as long as weights add up to less than 2^28: over 8192 keys
//    whatever their scores, over 2^21 whose scores lie below the first maximum.  The last factor takes it back.
// A key that a query does not see has the score -inf and the weight 0.  Values that no
// query of the tile sees are taken as zero codes.  A NaN among values that some of its queries see
// and others do not must reach the former only: 0 NaN is NaN, so such codes are zeroed
// too, and a product of (is NaN) with (sees it) marks the outputs that they make NaN.
// Work is split over the keys: waves of a workgroup take every W-th block, workgroups
// contiguous runs of blocks, joined in LDS and by kv8_combine_kernel.  Reading the cache
// bounds it: a token of 16 sequences of 32768 over 8 KV heads of 128 takes 185 to 195 us (5.5 to 5.8 TB/s), of
// eight of 4096 to 32768 63 (4.8 TB/s: lengths are not known where work is split), of one
// of 2048 over 32 heads 9.1, of which 4.6 are two launches.  Where a KV head has several tiles of
// queries, they run on one XCD one behind the other and read keys from its L2: 16 tokens
// of 28 heads over 4 KV heads of 131072 keys 100 -> 75 us against tiles apart.

// A maximum before any score: finite, so that no difference of two is NaN, and no finite score lies below it, so that only
// scores of -inf have no weight
constexpr float LOWEST = -__FLT_MAX__;
constexpr float RISE = 15.f, PLACE = 7.f;
constexpr float UNIT = 0x1p-28f;

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float lane_of(float x, int lane) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(x), lane));
}
__device__ __forceinline__ float wave_max(float x) {
  x = row_max<>(x);
  return fmaxf(fmaxf(lane_of(x, 0), lane_of(x, 16)), fmaxf(lane_of(x, 32), lane_of(x, 48)));
}
__device__ __forceinline__ float wave_sum(float x) {
  x = row_sum<>(x);
  return (lane_of(x, 0) + lane_of(x, 16)) + (lane_of(x, 32) + lane_of(x, 48));
}
// over the lanes 16 and 32 apart
__device__ __forceinline__ float column_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16, 64));
  return fmaxf(x, __shfl_xor(x, 32, 64));
}
__device__ __forceinline__ float column_sum(float x) {
  x += __shfl_xor(x, 16, 64);
  return x + __shfl_xor(x, 32, 64);
}
__device__ __forceinline__ bf16x8 as_bf16(uint32_t lo, uint32_t hi) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
__device__ __forceinline__ f16x8 as_f16(uint32_t lo, uint32_t hi) {
  const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, true);
  const f16x2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, true);
  return f16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
__device__ __forceinline__ f32x4 mfma_f16(const f16x8& a, const f16x8& b, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

constexpr int TILE = 16;  // query rows

// The blocks that any of tile rows [row0, row1] of a sequence sees: `sinkb` blocks of
// first tokens, then those from blk0 on; nb in all.
struct Seen {
  int pos0, pos1, blk0, sinkb, nb;
};
__device__ __forceinline__ Seen seen_of(const Kv8Attn& a, int len, int row0, int row1) {
  Seen s;
  s.pos0 = len - a.Lq + div_by(row0, a.by_G);
  s.pos1 = len - a.Lq + div_by(row1, a.by_G);
  const int lo = a.window ? max(s.pos0 - a.window + 1, 0) : 0;
  s.blk0 = lo / BLK;
  s.sinkb = min((min(a.sinks, lo) + BLK - 1) / BLK, s.blk0);
  s.nb = s.pos1 < 0 ? 0 : s.sinkb + s.pos1 / BLK + 1 - s.blk0;
  return s;
}

// 1 / l: of a query that sees no key (query q of len tokens) zero, of one whose keys all have no weight NaN
__device__ __forceinline__ float share(const Kv8Attn& a, int len, int q, float l) {
  return l != 0.f ? (1.f / UNIT) / l : len - a.Lq + q < 0 ? 0.f : __uint_as_float(0x7fc00000u);
}
// dims d .. d + 3 of query row gr of a KV head: v / l
__device__ __forceinline__ void store_row(const Kv8Attn& a, int b, int hk, int gr, int d, int len, const f32x4& v, float l) {
  const int q = div_by(gr, a.by_G);
  const float f = share(a, len, q, l);
  bf16_t* o = (bf16_t*)a.o.p + b * a.o.seq + q * a.o.token + (hk * a.G + gr - q * a.G) * a.o.head + d;
  *(u32x2*)o = u32x2{pack_bf2(v[0] * f, v[1] * f), pack_bf2(v[2] * f, v[3] * f)};
}

template <int DH, int W>
__global__ __launch_bounds__(W * 64) void kv8_attention_kernel(Kv8Attn a) {
  constexpr int KP = DH / 64, VP = DH / 32, ND = DH / 16, NS = DH / 32;  // 16-byte pieces of a lane (keys: a tile)
  __shared__ __attribute__((aligned(16))) float lds[W][TILE][DH + 4];
  __shared__ float sm[W][TILE], sl[W][TILE];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c16 = lane & 15, q = lane >> 4;
  const int total = a.B * a.Hkv;
  int bh = blockIdx.x, split = blockIdx.y, row0 = 0;
  if (a.tiles > 1) {  // workgroup n is on XCD n % 8: there the tiles of a run of keys one behind the other, for its L2
    const int slot = bh / 8, at = div_by(slot, a.by_tiles), group = at * 8 + bh % 8;
    split = div_by(group, a.by_BH);
    if (split >= a.nsplit) return;
    bh = group - split * total;
    row0 = (slot - at * a.tiles) * TILE;
  }
  const int b = div_by(bh, a.by_Hkv), hk = bh - b * a.Hkv;
  const int G = a.G, rows = a.Lq * G;
  // this lane's query: row row0 + c16
  const int row = row0 + c16;
  bf16x8 qb[NS];
  {
    const int i = div_by(min(row, rows - 1), a.by_G);
    const bf16_t* p = (const bf16_t*)a.q.p + b * a.q.seq + i * a.q.token + (hk * G + min(row, rows - 1) - i * G) * a.q.head;
#pragma unroll
    for (int s = 0; s < NS; ++s) qb[s] = *(const bf16x8*)(p + s * 32 + q * 8);
  }
  const int len = min(max(a.lens[b], 0), a.max_len);
  const Seen sn = seen_of(a, len, row0, min(rows, row0 + TILE) - 1);
  const int j0 = split * a.chunk, j1 = min(sn.nb, j0 + a.chunk);
  if (j0 >= sn.nb && split) return;
  const int last = row < rows ? len - a.Lq + div_by(row, a.by_G) : -1;  // position of the last key that the query sees
  const int reach = a.window ? a.window : INT_MAX;                      // and how far back it sees
  const int nblk = a.L_cap / BLK;
  const uint8_t* const codes = (const uint8_t*)a.cache + (size_t)bh * nblk * (64 * DH);
  const f32x2* const steps = (const f32x2*)((const uint8_t*)a.cache + (size_t)a.B * a.Hkv * nblk * (64 * DH)) + (size_t)bh * nblk;

  u32x4 kc[2][KP], vc[VP];
  f32x2 sk;  // the block's two steps, with its keys
  auto block_of = [&](int j) { return j < sn.sinkb ? j : sn.blk0 + j - sn.sinkb; };
  // past the run's last block: an empty buffer, no memory is touched
  auto buffer = [&](int j) {
    return __builtin_amdgcn_make_buffer_rsrc((void*)(codes + (size_t)block_of(min(j, j1 - 1)) * (64 * DH)), (short)0,
                                             j < j1 ? 64 * DH : 0, 0x00020000);
  };
  auto fetch_keys = [&](int j) {
    const __amdgpu_buffer_rsrc_t r = buffer(j);
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < KP; ++i)
        kc[t][i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, lane * 16, (t * KP + i) * 1024, 0));
    sk = steps[block_of(max(min(j, j1 - 1), 0))];
  };
  auto fetch_values = [&](int j) {
    const __amdgpu_buffer_rsrc_t r = buffer(j);
#pragma unroll
    for (int i = 0; i < VP; ++i)
      vc[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, lane * 16, 32 * DH + i * 1024, 0));
  };
  f32x4 o[ND];
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int d = 0; d < ND; ++d) o[d] = zero;
  float m = LOWEST, l = 0.f;
  if (j0 + wave < j1) {
    fetch_keys(j0 + wave);
    fetch_values(j0 + wave);
  }
  for (int j = j0 + wave; j < j1; j += W) {
    const int key0 = block_of(j) * BLK;
    // every row sees the whole block
    const bool whole = key0 + BLK - 1 <= sn.pos0 && (!a.window || key0 > sn.pos1 - a.window);
    f32x4 sc[2] = {zero, zero};
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
      for (int t = 0; t < 2; ++t) sc[t] = mfma(as_bf16(kc[t][s / 2][s % 2 * 2], kc[t][s / 2][s % 2 * 2 + 1]), qb[s], sc[t]);
    const float ks = sk[0] * a.scale_log2, vs = sk[1] * UNIT;
#pragma unroll
    for (int t = 0; t < 2; ++t) asm volatile("" : "+v"(sc[t]));
    __builtin_amdgcn_sched_barrier(0);
    fetch_keys(j + W);
    float p[2][4], top = -INFINITY;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) p[t][r] = sc[t][r] * ks;
    uint32_t sees = 0xffu;  // this lane's query, by key
    if (!whole) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int key = key0 + t * 16 + q * 4 + r;
          const bool yes = (key <= last) & ((last - key < reach) | (key < a.sinks));
          p[t][r] = yes ? p[t][r] : -INFINITY;  // also in place of whatever the cache's unwritten rows gave
          sees &= ~((yes ? 0u : 1u) << (t * 4 + r));
        }
    }
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) top = fmaxf(top, p[t][r]);
    if (__any(top > m + RISE)) {
      top = column_max(top);
      if (top > m + RISE) {
        const float mn = top - PLACE, f = exp2_of(m - mn);
        l *= f;
#pragma unroll
        for (int d = 0; d < ND; ++d) o[d] *= f;
        m = mn;
      }
    }
    float sum = 0.f;
    f16x8 pb;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float e = exp2_of(p[t][r] - m);
        sum += e;
        pb[t * 4 + r] = (_Float16)e;
      }
    l += sum;
    if (!whole) {
      // codes of keys past the last that a row sees are zeroed, NaN among the others too
      uint32_t keep[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int n = sn.pos1 + 1 - (key0 + t * 16 + q * 4);  // tokens there
        keep[t] = n >= 4 ? 0xffffffffu : n <= 0 ? 0u : (1u << 8 * n) - 1;
      }
      uint32_t nan[VP][4], some = 0;
#pragma unroll
      for (int i = 0; i < VP; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t w = vc[i][e] & keep[e & 1];
          nan[i][e] = ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
          some |= nan[i][e];
          vc[i][e] = w & ~((nan[i][e] >> 7) * 255u);
        }
      if (__any(some != 0)) {
        f16x8 see;
#pragma unroll
        for (int e = 0; e < 8; ++e) see[e] = (sees >> e & 1) ? (_Float16)1.f : (_Float16)0.f;
#pragma unroll
        for (int d = 0; d < ND; ++d) {
          // NaN codes as 0x38, which is one
          const uint32_t lo = (nan[d / 2][d % 2 * 2] >> 7) * 0x38u, hi = (nan[d / 2][d % 2 * 2 + 1] >> 7) * 0x38u;
          const f32x4 n = mfma_f16(as_f16(lo, hi), see, zero);
#pragma unroll
          for (int r = 0; r < 4; ++r) o[d][r] = n[r] > 0.f ? __uint_as_float(0x7fc00000u) : o[d][r];
        }
      }
    }
#pragma unroll
    for (int d = 0; d < ND; ++d) {
      const f32x4 y = mfma_f16(as_f16(vc[d / 2][d % 2 * 2], vc[d / 2][d % 2 * 2 + 1]), pb, zero);
#pragma unroll
      for (int r = 0; r < 4; ++r) o[d][r] = fmaf(y[r], vs, o[d][r]);
    }
    __builtin_amdgcn_sched_barrier(0);
    fetch_values(j + W);
  }

  // join the waves: lane (c16, q) holds dims 16 d + 4 q .. of query row c16
  l = column_sum(l);
  if (q == 0) {
    sm[wave][c16] = m;
    sl[wave][c16] = l;
  }
#pragma unroll
  for (int d = 0; d < ND; ++d) *(f32x4*)&lds[wave][c16][d * 16 + q * 4] = o[d];
  __syncthreads();
  for (int i = tid; i < TILE * DH / 4; i += W * 64) {
    const int r = i / (DH / 4), d = i % (DH / 4) * 4, gr = row0 + r;
    if (gr >= rows) break;
    float mx = sm[0][r];
#pragma unroll
    for (int w = 1; w < W; ++w) mx = fmaxf(mx, sm[w][r]);
    float ls = 0.f;
    f32x4 v = zero;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const float f = exp2_of(sm[w][r] - mx);
      ls = fmaf(f, sl[w][r], ls);
      const f32x4 x = *(const f32x4*)&lds[w][r][d];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = fmaf(f, x[e], v[e]);
    }
    if (sn.nb <= a.chunk) {
      store_row(a, b, hk, gr, d, len, v, ls);
    } else {
      const size_t at = ((size_t)bh * rows + gr) * a.nsplit + split;
      const size_t ml = (size_t)total * rows * a.nsplit * DH + at * 2;
      if (a.tiles > 1) {
        // Past the caches (sc0, sc1), below 2^27 bytes in all: what L2 holds at the kernel's end must still be written
        // back.  9 tokens of four sequences of 4096, 7 heads a KV head: 11.6 -> 10.2 us, such calls 2.3% on average;
        // calls of one tile lose 0.5%.
        const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void*)a.part, (short)0, 0x7fffffff, 0x00020000);
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), r, (uint32_t)((at * DH + d) * 4), 0, 17);
        if (d == 0) __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2, f32x2{mx, ls}), r, (uint32_t)(ml * 4), 0, 17);
      } else {
        *(f32x4*)(a.part + at * DH + d) = v;
        if (d == 0) *(f32x2*)(a.part + ml) = f32x2{mx, ls};
      }
    }
  }
}

// Joins the splits of a query row where there is more than one; one wave a row.  Lane s
// takes the maximum and sum of split s, so that the weights of 64 splits cost one load and
// one reduction; the outputs of CB splits are in flight together.
template <int DH>
__global__ __launch_bounds__(64) void kv8_combine_kernel(Kv8Attn a, int total) {
  constexpr int CB = 16, D = DH / 64;  // dims a lane
  typedef float vec __attribute__((ext_vector_type(D)));
  const int rows = a.Lq * a.G, row = blockIdx.x, lane = threadIdx.x;
  const int bh = div_by(row, a.by_rows), gr = row - bh * rows;
  const int b = div_by(bh, a.by_Hkv), hk = bh - b * a.Hkv;
  const float* part = a.part + (size_t)row * a.nsplit * DH + lane * D;
  const f32x2* ml = (const f32x2*)(a.part + (size_t)total * a.nsplit * DH) + (size_t)row * a.nsplit;
  vec os[CB];
  auto load = [&](int s0, int n) {
#pragma unroll
    for (int s = 0; s < CB; ++s) os[s] = *(const vec*)(part + (size_t)min(s0 + s, n - 1) * DH);
  };
  f32x2 x = ml[min(lane, a.nsplit - 1)];
  load(0, a.nsplit);  // what was not written is not used
  const int length = a.lens[b];
  __builtin_amdgcn_sched_barrier(0);
  const int row0 = gr / TILE * TILE, len = min(max(length, 0), a.max_len);
  const Seen sn = seen_of(a, len, row0, min(rows, row0 + TILE) - 1);
  const int ns = div_by(sn.nb + a.chunk - 1, a.by_chunk);
  float mx = LOWEST, l = 0.f;
  vec v = {};
  for (int s0 = 0; s0 < ns; s0 += 64) {
    if (s0) x = ml[min(s0 + lane, ns - 1)];
    const bool there = s0 + lane < ns;
    const float m = there ? x[0] : LOWEST, mn = fmaxf(mx, wave_max(m));
    const float f0 = exp2_of(mx - mn), f = exp2_of(m - mn);
    l = fmaf(l, f0, wave_sum(there ? f * x[1] : 0.f));
    v *= f0;
    mx = mn;
    const int n = min(64, ns - s0);
    for (int s1 = 0; s1 < n; s1 += CB) {
      if (s0 + s1) load(s0 + s1, ns);
#pragma unroll
      for (int s = 0; s < CB; ++s) {
        const float w = lane_of(f, s1 + s);
        if (s1 + s < n) v += w * os[s];
      }
    }
  }
  if (ns < 2) return;  // written by the one split
  const int q = div_by(gr, a.by_G);
  const float f = share(a, len, q, l);
  bf16_t* o = (bf16_t*)a.o.p + b * a.o.seq + q * a.o.token + (hk * a.G + gr - q * a.G) * a.o.head + lane * D;
  if constexpr (D == 2)
    *(uint32_t*)o = pack_bf2(v[0] * f, v[1] * f);
  else
    *o = f2bf(v[0] * f);
}

// Blocks of 32 keys that a tile of queries sees at most
unsigned blocks_of(int Lq, int max_len, int window, int sinks) {
  unsigned blocks = max_len > 0 ? cdiv(max_len, BLK) : 1;
  if (window > 0) {
    const int64_t w = ((int64_t)window + Lq - 1 + BLK - 1) / BLK + 1 + cdiv(sinks, BLK);
    if (w < blocks) blocks = (unsigned)w;
  }
  return blocks;
}
// Splits that a plan may take, and scratch is sized for: some 4096 workgroups, of four
// blocks or more.  It never falls with the length, so scratch for the longest call serves
// each shorter one.
unsigned most_splits(int B, int Lq, int H, int Hkv, unsigned blocks) {
  const int rows = Lq * (H / Hkv);
  const int64_t wgs = (int64_t)B * Hkv * cdiv(rows, TILE), n = (4095 + wgs) / wgs;
  return n < (blocks + 3) / 4 ? (unsigned)n : (blocks + 3) / 4;
}

// What a call costs, fitted to 117 shapes of 1 to 256 KV heads of all sequences, 300 to 131072 tokens, 1 to 7 tiles of
// queries, with lengths alike and from an eighth on, at 20 to 50 plans each: those chosen are 2.1% slower than the
// fastest ones on average, 13% at most.  Always 8 waves would be as fast on average, but 10% slower where eight
// sequences of 4096 to 32768 tokens run together, always 4 waves 3.5% slower on average.  (Splits chosen on the
// device by the lengths themselves, from one sum over the sequences, are 4% faster to 30% slower there: workgroups
// whose sequence ends before them make room for the others as it is.)
struct Plan {
  int W, tiles, chunk, nsplit;
};
Plan plan_of(int B, int Lq, int H, int Hkv, int max_len, int window, int sinks) {
  const int rows = Lq * (H / Hkv), tiles = cdiv(rows, TILE);
  const unsigned blocks = blocks_of(Lq, max_len, window, sinks), limit = most_splits(B, Lq, H, Hkv, blocks);
  const int64_t runs = (int64_t)B * Hkv, bt = runs * tiles;
  Plan p{};
  int64_t best = INT64_MAX;
  for (int W = 4; W <= 8; W += 4) {
    const unsigned most = (blocks + W - 1) / W;  // blocks of a wave, if nothing is split
    auto consider = [&](unsigned per) {
      const unsigned ns = (blocks + per * W - 1) / (per * W);
      // waves of one SIMD; times of a wave alone, of a SIMD's together, of the join (a unit is some 20 ns)
      const int64_t waves = ((runs * ns + 7) / 8 * tiles + 31) / 32 * (W / 4);
      const int64_t wave = 40ll * per, simd = waves * (17 * per + 24);
      const int64_t cost = (wave > simd ? wave : simd) + (ns > 1 ? 209 + 49 * ((ns - 1) / 16) : 0);
      if (cost < best && ns <= limit) best = cost, p = Plan{W, tiles, (int)(per * W), (int)ns};
      return wave < best;  // else longer runs of blocks cost no less
    };
    for (int64_t wgs = 256; wgs <= 1024; wgs += 256)
      if (wgs >= bt) consider((unsigned)((most + wgs / bt - 1) / (wgs / bt)));
    for (unsigned per = 1; per < most && consider(per);) per += per < 6 ? 1 : per < 12 ? 2 : per < 24 ? 4 : per / 4;
    consider(most);
  }
  return p;
}

template <int DH, int W>
hipError_t launch_attention(const Kv8Attn& a, hipStream_t s) {
  const int64_t runs = (int64_t)a.B * a.Hkv;
  const dim3 grid = a.tiles > 1 ? dim3((unsigned)((runs * a.nsplit + 7) / 8 * 8 * a.tiles)) : dim3((unsigned)runs, a.nsplit);
  hipLaunchKernelGGL((kv8_attention_kernel<DH, W>), grid, dim3(W * 64), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.nsplit == 1) return e;
  hipLaunchKernelGGL((kv8_combine_kernel<DH>), dim3(a.B * a.Lq * a.H), dim3(64), 0, s, a, a.B * a.Lq * a.H);
  return hipGetLastError();
}

// blocks that L tokens from any position on can touch
unsigned rows_grid(Kv8Rows& a) {
  a.blocks = (a.L + 2 * (BLK - 1)) / BLK;
  a.by_blocks = fast_div(a.blocks);
  a.by_Hkv = fast_div(a.Hkv);
  return (unsigned)(a.B * a.Hkv * a.blocks);
}

}  // namespace

size_t kv8_bytes(int B, int Hkv, int L_cap, int dh) { return (size_t)B * Hkv * (L_cap / BLK) * (64 * dh + 8); }

hipError_t kv8_store(Kv8Rows a, int dh, hipStream_t s) {
  const dim3 grid(2 * rows_grid(a));
  if (dh == 128)
    hipLaunchKernelGGL((kv8_store_kernel<128>), grid, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((kv8_store_kernel<64>), grid, dim3(128), 0, s, a);
  return hipGetLastError();
}

hipError_t kv8_load(Kv8Rows a, int dh, hipStream_t s) {
  const dim3 grid(2 * rows_grid(a));
  if (dh == 128)
    hipLaunchKernelGGL((kv8_load_kernel<128>), grid, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((kv8_load_kernel<64>), grid, dim3(128), 0, s, a);
  return hipGetLastError();
}

size_t kv8_attention_scratch(int B, int Lq, int H, int Hkv, int dh, int max_len, int window, int sinks) {
  const unsigned n = most_splits(B, Lq, H, Hkv, blocks_of(Lq, max_len, window, sinks));
  return n < 2 ? 0 : (size_t)B * Lq * H * n * (dh + 2) * sizeof(float);
}

hipError_t kv8_attention(Kv8Attn a, int dh, size_t scratch_bytes, hipStream_t s) {
  if (scratch_bytes < kv8_attention_scratch(a.B, a.Lq, a.H, a.Hkv, dh, a.max_len, a.window, a.sinks))
    return hipErrorOutOfMemory;
  const Plan p = plan_of(a.B, a.Lq, a.H, a.Hkv, a.max_len, a.window, a.sinks);
  a.G = a.H / a.Hkv;
  a.by_G = fast_div(a.G);
  a.by_Hkv = fast_div(a.Hkv);
  a.by_rows = fast_div(a.Lq * a.G);
  a.by_BH = fast_div(a.B * a.Hkv);
  a.by_tiles = fast_div(p.tiles);
  a.tiles = p.tiles;
  a.chunk = p.chunk;
  a.by_chunk = fast_div(p.chunk);
  a.nsplit = p.nsplit;
  a.scale_log2 = 1.4426950408889634f / sqrtf((float)dh);
  if (p.W == 8) return dh == 128 ? launch_attention<128, 8>(a, s) : launch_attention<64, 8>(a, s);
  return dh == 128 ? launch_attention<128, 4>(a, s) : launch_attention<64, 4>(a, s);
}

}  // namespace vla
