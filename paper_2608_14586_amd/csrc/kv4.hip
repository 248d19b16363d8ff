// The KV cache in 4 bits: rows into it, rows out of it, and attention over it.
//
// Every 32 dims of a key or value row are one group of 16 levels: s = (max -
// min) * (1 / 15) in bf16, m = min (a bf16 number already), code = (x - m) / s
// to the nearest, ties to the even one; the row stands for m + s code.
//
// The cache of one sequence and KV head is a run of blocks of 32 tokens, 40 dh
// bytes each, everything that attention needs of them side by side:
//   key codes    [token 32][quarter 4][group dh/32] words: the 8 codes of dims
//                32 group + 8 quarter + j, code j in nibble j / 2 (even j) or
//                4 + j / 2 (odd j), the word then rotated left by 3
//   value codes  [quarter 4][d % 16][d / 16] words: the 8 codes of dim d of
//                tokens 4 quarter + i (nibble i) and 16 + 4 quarter + i (nibble
//                4 + i), i < 4, nibbles 3 and 7 exchanged, the word then rotated
//                left by 6
//   key params   [token 32][group] words: s in the low half, m in the high
//   value params [token 32][group] words
// In this order a wave's loads of keys and values are contiguous and every
// 32-bit word of codes is one lane's operand of an MFMA step, nibbles i and 4 +
// i two numbers of it.  Keys become bf16: rotated to the top mantissa bits (3-6)
// of 16.0 they are 16 + c, by one rotate and one and-or a pair; the layout saves
// the first pair its rotate.  Values become fp16, whose 10 bits of mantissa
// hold two nibbles: at bits 6-9 of 16.0 one is 16 + c, at bits 2-5 of 256.0 it is
// 256 + c, so one rotate by 8 serves all four pairs: 5 instructions a word in
// place of 7, 1 to 3% of attention's time.
#include <limits.h>

#include <type_traits>

#include "kernels.h"

namespace vla {
namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

constexpr uint32_t ONES = 0x3f803f80u;  // bf16 1.0 twice
constexpr int BLK = 32;  // tokens per block
constexpr float LOWEST = -3e38f;  // a maximum before any score: finite, so that no difference of two is NaN
constexpr float RAISE = 8.f;  // log2 by which scores may rise before the maximum follows
// exponents: P' as fp16 stays below 2^MOST, and the largest is put below 2^PLACE where it does not
constexpr int MOST = 15, PLACE = 7;
constexpr float MID = 7.5f;  // of the codes
constexpr int KROT = 3, VROT = 6;

// 8 codes of a word of value codes, constants in registers as in UnpackCodes:
// pairs 0 and 2 are 16 + c, pairs 1 and 3 256 + c
struct UnpackValues {
  uint32_t bias16 = 0x4c004c00u, mask16 = 0x03c003c0u, bias256 = 0x5c005c00u, mask256 = 0x003c003cu;
  __device__ __forceinline__ UnpackValues() {
    asm("" : "+s"(bias16), "+v"(mask16));
    asm("" : "+s"(bias256), "+v"(mask256));
  }
  __device__ __forceinline__ f16x8 operator()(uint32_t w) const {
    const uint32_t r = __builtin_amdgcn_alignbit(w, w, 8);
    const u32x4 v = {(w & mask16) | bias16, (r & mask256) | bias256, (r & mask16) | bias16, (w & mask256) | bias256};
    return __builtin_bit_cast(f16x8, v);
  }
};
__device__ __forceinline__ float lo16(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi16(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
using ::mfma;  // of bf16, beside the one of fp16
__device__ __forceinline__ f32x4 mfma(const f16x8& a, const f16x8& b, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// ------------------------------------------------------------ rows in and out

struct Group4 {
  uint32_t codes;   // of this lane's 8 dims
  uint32_t params;  // of the group
};
// The codes of 8 values whose group spans [lo, lo + d], with step s and its
// approximate inverse.  t = x - lo is rounded to fp32, as in plain fp32 code (lo
// = -2.5, s = 1, x = 2^-30: 2.5, code 2); from there on a code is t / s rounded once.
// The quotient is corrected once by its remainder.  Where t / s is a border k + 1/2
// between two codes it comes out exact.  Elsewhere t is at least one fp32 step from
// (k + 1/2) s, which has 13 bits, so t / s is off the border by 2^-24 of itself and
// more (s, of 8 bits, keeps t's mantissa from 2 by 2^-7), and rounding it to fp32
// takes less.  s lies within 2^-9 of d / 15, so none rounds to more than 15.
// Halves of a word are summed up in fp32, 16 bits each.
__device__ __forceinline__ uint32_t codes_of(const float (&x)[8], float lo, float s, float inv) {
  float half[2] = {0.f, 0.f};
#pragma unroll
  for (int e = 7; e >= 0; --e) {
    const float t = x[e] - lo;
    float q = t * inv;
    q = rintf(fmaf(fmaf(-q, s, t), inv, q));
    half[e & 1] = fmaf(half[e & 1], 16.f, q);
  }
  return (uint32_t)half[0] | (uint32_t)half[1] << 16;
}
// Quantises the 8 dims of this lane; the 4 lanes of a group hold its 32 dims.
__device__ __forceinline__ Group4 quantise(const u32x4& w) {
  float x[8], any = 0.f;  // any: a sum that is finite only if all values are
  const bf16x8 v = __builtin_bit_cast(bf16x8, w), one = __builtin_bit_cast(bf16x8, u32x4{ONES, ONES, ONES, ONES});
  any = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(v, v, 0, 1), __builtin_shufflevector(one, one, 0, 1), any, false);
  any = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(v, v, 2, 3), __builtin_shufflevector(one, one, 0, 1), any, false);
  any = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(v, v, 4, 5), __builtin_shufflevector(one, one, 0, 1), any, false);
  any = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(v, v, 6, 7), __builtin_shufflevector(one, one, 0, 1), any, false);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[2 * e] = lo16(w[e]);
    x[2 * e + 1] = hi16(w[e]);
  }
  float lo = x[0], hi = x[0];
#pragma unroll
  for (int e = 1; e < 8; ++e) {
    lo = fminf(lo, x[e]);
    hi = fmaxf(hi, x[e]);
  }
  lo = -row_max<4>(-lo);
  hi = row_max<4>(hi);
  any = row_sum<4>(any);
  const float d = hi - lo;
  const uint32_t m = __float_as_uint(lo) & 0xffff0000u;
  // where a value or a sum of values is not finite: once more with care
  if (!(fabsf(any) <= 3.4e38f && d <= 3.4e38f)) {
    uint32_t mag = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) mag = max(mag, max(w[e] & 0x7fffu, w[e] >> 16 & 0x7fffu));
    // of the group; the condition above is the same in its 4 lanes
    if (row_max<4>((float)mag) >= (float)0x7f80) return Group4{0u, 0x7fc07fc0u};  // the group reads as NaN
    if (!(d <= 3.4e38f)) {  // a range past fp32: everything by halves
      const float half = 0.5f * hi - 0.5f * lo;
      const uint16_t sb = f2bf(half / 7.5f);
      const float hs = 0.5f * bf2f(sb);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] *= 0.5f;
      return Group4{codes_of(x, 0.5f * lo, hs, 1.f / hs), m | sb};
    }
  }
  if (!(d >= 0x1p-99f)) return Group4{0u, m};
  // by 1 / 15 in fp32: within 2^-24 of d / 15, which decides only quotients that
  // lie between two bf16 numbers
  const uint16_t sb = f2bf(d * (1.f / 15));
  const float s = bf2f(sb);
  return Group4{codes_of(x, lo, s, __builtin_amdgcn_rcpf(s)), m | sb};
}

// Transposes 8 x 8 codes of 4 bits: nibble c of word r becomes nibble r of word c.
__device__ __forceinline__ void transpose8(uint32_t (&w)[8]) {
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const uint32_t a = w[r], b = w[r + 4];
    w[r] = __builtin_amdgcn_perm(b, a, 0x05040100u);
    w[r + 4] = __builtin_amdgcn_perm(b, a, 0x07060302u);
  }
#pragma unroll
  for (int r = 0; r < 8; r += r % 2 ? 3 : 1) {
    const uint32_t a = w[r], b = w[r + 2];
    w[r] = __builtin_amdgcn_perm(b, a, 0x06020400u);
    w[r + 2] = __builtin_amdgcn_perm(b, a, 0x07030501u);
  }
#pragma unroll
  for (int r = 0; r < 8; r += 2) {
    const uint32_t a = w[r], b = w[r + 1];
    w[r] = (a & 0x0f0f0f0fu) | (b << 4 & 0xf0f0f0f0u);
    w[r + 1] = (a >> 4 & 0x0f0f0f0fu) | (b & 0xf0f0f0f0u);
  }
}
// dim 8 j + e of a token is code nibble_of(e) of its word j
__host__ __device__ constexpr int nibble_of(int e) { return e / 2 + (e & 1) * 4; }
__host__ __device__ constexpr int dim_of(int nibble) { return nibble % 4 * 2 + nibble / 4; }
// nibble i of a quarter's value codes is token token_of(quarter, i) of the block
__device__ __forceinline__ int token_of(int quarter, int i) {
  return 4 * quarter + i % 4 + (i % 4 == 3 ? 1 - i / 4 : i / 4) * 16;
}

// this workgroup's block of the cache and the tokens of the call in it:
// tokens [t0, t1) of the block are tokens from + (t - t0) of the sequence's rows
struct Span {
  int b, h, blk, t0, t1, from;
};
__device__ __forceinline__ Span span_of(const Kv4Rows& a, int wg) {
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

// One workgroup for the keys of a block of 32 tokens of a head (even ones) or
// for its values; DH / 8 lanes a row.  About 110 instructions a lane and 8
// values take as long as the memory does, so there are workgroups enough for
// two rounds, whose loads and arithmetic overlap.  The value codes cross LDS
// to the threads that hold 8 dims of 8 tokens and transpose them.  2048 tokens of
// 32 heads, dh = 128 (44 MB): 12.2 us where they lie in the 256 MB cache, 3.6 TB/s
// (9.7 with the arithmetic left out), from memory 14.4.
template <int DH>
__global__ __launch_bounds__(256) void kv4_store_kernel(Kv4Rows a) {
  constexpr int LPR = DH / 8, RPP = 256 / LPR, P = BLK / RPP, NG = DH / 32, ND = DH / 16;  // lanes a row, rows a pass
  __shared__ uint32_t vs[BLK][LPR];
  const Span s = span_of(a, blockIdx.x >> 1);
  const bool values = blockIdx.x & 1;
  if (s.t0 >= s.t1) return;
  uint8_t* base = (uint8_t*)a.cache + (((size_t)s.b * a.Hkv + s.h) * (a.L_cap / BLK) + s.blk) * (40 * DH);
  const int tid = threadIdx.x, j = tid % LPR, g = j / 4, kq = j % 4;
  const Heads& in = values ? a.v : a.k;
  u32x4 x[P];
#pragma unroll
  for (int r = 0; r < P; ++r) {
    const int t = r * RPP + tid / LPR;
    if (t >= s.t0 && t < s.t1)
      x[r] = *(const u32x4*)((const bf16_t*)in.p + s.b * in.seq + (int64_t)(s.from + t - s.t0) * in.token +
                             s.h * in.head + j * 8);
  }
  uint32_t* vc = (uint32_t*)(base + 16 * DH);
  auto word_at = [&](int c) {  // of value code words of quarter tid / LPR
    const int d = j * 8 + dim_of(c);
    return (tid / LPR * 16 + d % 16) * ND + d / 16;
  };
  uint32_t old[8];  // of a block that the call does not fill
  if (values && s.t1 - s.t0 < BLK && tid < 4 * LPR)
#pragma unroll
    for (int c = 0; c < 8; ++c) old[c] = vc[word_at(c)];
#pragma unroll
  for (int r = 0; r < P; ++r) {
    const int t = r * RPP + tid / LPR;
    if (t < s.t0 || t >= s.t1) continue;
    const Group4 q = quantise(x[r]);
    if (values)
      vs[t][j] = q.codes;
    else
      *(uint32_t*)(base + t * (DH / 2) + kq * (DH / 8) + g * 4) = rotl(q.codes, KROT);
    if (kq == 0) *(uint32_t*)(base + (values ? 36 : 32) * DH + (t * NG + g) * 4) = q.params;
  }
  if (!values) return;
  __syncthreads();
  if (tid >= 4 * LPR) return;
  const int q4 = tid / LPR;
  uint32_t w[8], have = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int t = token_of(q4, i);
    const bool there = t >= s.t0 && t < s.t1;
    w[i] = there ? vs[t][j] : 0u;
    have |= there ? 15u << 4 * i : 0u;
  }
  if (have == 0) return;
  transpose8(w);
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    if (have != 0xffffffffu) w[c] |= rotl(old[c], 32 - VROT) & ~have;  // tokens of other calls keep theirs
    vc[word_at(c)] = rotl(w[c], VROT);
  }
}

// The inverse: 4 DH / 8 threads transpose the block's value codes into LDS,
// word j of every token as the keys have it.  8.4 us for the same 44 MB, 5.2 TB/s, and
// 14.0 where the cache is read from memory and the rows go there.
template <int DH>
__global__ __launch_bounds__(256) void kv4_load_kernel(Kv4Rows a) {
  constexpr int LPR = DH / 8, RPP = 256 / LPR, P = BLK / RPP, NG = DH / 32, ND = DH / 16;
  __shared__ uint32_t vs[BLK][LPR];
  const Span s = span_of(a, blockIdx.x);
  if (s.t0 >= s.t1) return;
  const uint8_t* base = (const uint8_t*)a.cache + (((size_t)s.b * a.Hkv + s.h) * (a.L_cap / BLK) + s.blk) * (40 * DH);
  const int tid = threadIdx.x, j = tid % LPR, g = j / 4, kq = j % 4;
  uint32_t kw[P], prm[2][P];
#pragma unroll
  for (int r = 0; r < P; ++r) {
    const int t = r * RPP + tid / LPR;
    kw[r] = *(const uint32_t*)(base + t * (DH / 2) + kq * (DH / 8) + g * 4);
#pragma unroll
    for (int p = 0; p < 2; ++p) prm[p][r] = *(const uint32_t*)(base + (p ? 36 : 32) * DH + (t * NG + g) * 4);
  }
  if (tid < 4 * LPR) {
    const int q4 = tid / LPR;
    uint32_t w[8];
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      const int d = j * 8 + dim_of(c);
      w[c] = rotl(((const uint32_t*)(base + 16 * DH))[(q4 * 16 + d % 16) * ND + d / 16], 32 - VROT);
    }
    transpose8(w);
#pragma unroll
    for (int i = 0; i < 8; ++i) vs[token_of(q4, i)][j] = w[i];
  }
  __syncthreads();
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    const Heads& out = p ? a.v : a.k;
#pragma unroll
    for (int r = 0; r < P; ++r) {
      const int t = r * RPP + tid / LPR;
      if (t < s.t0 || t >= s.t1) continue;
      const uint32_t w = p ? vs[t][j] : rotl(kw[r], 32 - KROT);
      const float sc = lo16(prm[p][r]), mn = hi16(prm[p][r]);
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = fmaf(sc, (float)(w >> 4 * nibble_of(e) & 15u), mn);
      bf16_t* row = (bf16_t*)out.p + s.b * out.seq + (int64_t)(s.from + t - s.t0) * out.token + s.h * out.head;
      *(u32x4*)(row + j * 8) =
          u32x4{pack_bf2(x[0], x[1]), pack_bf2(x[2], x[3]), pack_bf2(x[4], x[5]), pack_bf2(x[6], x[7])};
    }
  }
}

// -------------------------------------------------------------- attention
//
// A decode step's attention reads each visible key and value once for the few
// queries that share its KV head, so it is bound by the cache's bytes, and by
// the instructions that turn codes into operands, which come close behind.
//  * scores: two codes become bf16 numbers 16 + c by a rotate and an and-or, so
//      q . k = sum_g [ s_g (sum (16 + c) q - 16 sum q) + m_g sum q ]
//    over the groups g of 32 dims: one MFMA step a group (queries against 16
//    keys), whose accumulators start from -16 sum q, and two multiply-adds in
//    fp32; sum q is a constant of the loop.
//  * softmax: a running maximum and sum per query, in fp32, one pass.
//  * values: with P the weights, per group P' = P s_g and b = 16 or 256 by the key,
//      sum P v = sum P' (b + c) - sum (b + 7.5) P' + sum P (m_g + 7.5 s_g)
//    the first sum by MFMA, the others in fp32 in the lane that holds P.  P' is
//    rounded to fp16, in a unit of each query and group of its own: a power of
//    two that puts the largest P' of the keys so far that this query sees between
//    2^6 and 2^15.  So a key weighs in a query's unit by what it adds to that query, and
//    one that the query does not see, or gives no weight, moves nothing, however
//    large its values.  The second sum is of the rounded P', so that rounding costs
//    2^-11 of at most 7.5 s_g P a key, a sixteenth of what a bf16 result's rounding
//    takes of 15 s_g P, and less than 2^-31 of the largest P' where P' is subnormal.
//    (Without the 7.5, the middle of the codes, it would be twice that, for 8 of 220
//    instructions; in bf16 eight times; hi and lo bf16 parts cost 12 instructions
//    a row and group against 6.)
// The 4 R queries of a tile sit in the MFMA rows 4 i + r, r < R, so with up to
// four of them a lane holds one useful score a key and not four (R = 1).
// P crosses from score lanes (one key each) to operand lanes (8 keys of one
// query) through LDS, as 32-bit pairs of the keys t and t + 16: that pairing
// is why the value codes of those tokens share a word's halves.
// More than 16 queries a KV head unpack the cache once for each 16 and less: 2048
// tokens, 32 heads over 8, one token's queries 6.2 us, 16 tokens' 12, 256 tokens' 34.
// Work is split over the keys: waves of a workgroup take every W-th block of
// 32 keys, workgroups contiguous runs of them, joined in LDS and by
// kv4_combine_kernel.
// With R = 1 and dh = 128 a block is about 220 vector instructions and 16 MFMAs
// a wave against 5120 bytes.  A wave alone on its SIMD takes 0.8 us a block that
// lies in cache and 1.2 from memory, two side by side 1.1 and 1.9: the memory
// comes first.  159 registers leave three waves a SIMD; two took a third longer
// over long caches, and four spill.  Eight sequences of up to 32768 tokens (32
// heads, 8 KV heads, 189 MB) take 42.7 us, 4.4 TB/s, joining and ragged ends
// included; one of 2049 tokens (32 KV heads) 7.5 us where it lies in the 256 MB
// cache and 8.8 from memory, of which two launches are 4.6.
// The loads of the next block go out in two parts, each into the registers that
// the part of this block before it has used up, unconditionally and below a
// scheduling barrier: with branches around them, or with a use of the old values
// left below them, the compiler waits for every load at the loop's end, which
// cost 2% of a long cache's time and 10% of short ones'.  A second block ahead
// gains nothing there and costs a wave a SIMD (43 -> 55 us).

// a value of one lane, for all
__device__ __forceinline__ float lane_of(float x, int lane) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(x), lane));
}
// over the wave
__device__ __forceinline__ float wave_max(float x) {
  x = row_max<>(x);
  return fmaxf(fmaxf(lane_of(x, 0), lane_of(x, 16)), fmaxf(lane_of(x, 32), lane_of(x, 48)));
}
__device__ __forceinline__ float wave_sum(float x) {
  x = row_sum<>(x);
  return (lane_of(x, 0) + lane_of(x, 16)) + (lane_of(x, 32) + lane_of(x, 48));
}

template <int N>
struct Words {
  uint32_t w[N];
};
// N words at byte `at` (this lane's) + `base` (the wave's) of a buffer
template <int N>
__device__ __forceinline__ Words<N> load_words(__amdgpu_buffer_rsrc_t r, uint32_t at, uint32_t base) {
  Words<N> x;
  if constexpr (N % 4 == 0) {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      const u32x4 v = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, at + 16 * i, base, 0));
#pragma unroll
      for (int e = 0; e < 4; ++e) x.w[4 * i + e] = v[e];
    }
  } else {
    const u32x2 v = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(r, at, base, 0));
    x.w[0] = v[0];
    x.w[1] = v[1];
  }
  return x;
}

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

// the largest of a row's 16 lanes, as whole numbers
__device__ __forceinline__ uint32_t row_max_u(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xf, 0xf, true));
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xf, 0xf, true));
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x141, 0xf, 0xf, true));
  return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x140, 0xf, 0xf, true));
}

// 1 / x of a power of two from 2^-126 to 2^126
__device__ __forceinline__ float inverse2(float x) { return __uint_as_float(0x7f000000u - __float_as_uint(x)); }

// The blocks that any of tile rows [row0, row1] of a sequence sees: `sinkb`
// blocks of first tokens, then those from blk0 on; nb in all.
struct Seen {
  int pos0, pos1, blk0, sinkb, nb;
};
__device__ __forceinline__ Seen seen_of(const Kv4Attn& a, int len, int row0, int row1) {
  Seen s;
  s.pos0 = len - a.Lq + div_by(row0, a.by_G);
  s.pos1 = len - a.Lq + div_by(row1, a.by_G);
  const int lo = a.window ? max(s.pos0 - a.window + 1, 0) : 0;
  s.blk0 = lo / BLK;
  s.sinkb = min((min(a.sinks, lo) + BLK - 1) / BLK, s.blk0);
  s.nb = s.pos1 < 0 ? 0 : s.sinkb + s.pos1 / BLK + 1 - s.blk0;
  return s;
}

// dims d .. d + 3 of query row gr of a KV head: v / l, zeros where no key was seen
__device__ __forceinline__ void store_row(const Kv4Attn& a, int b, int hk, int gr, int d, const f32x4& v, float l) {
  const int q = div_by(gr, a.by_G);
  const float f = l == 0.f ? 0.f : 1.f / l;
  bf16_t* o = (bf16_t*)a.o.p + b * a.o.seq + q * a.o.token + (hk * a.G + gr - q * a.G) * a.o.head + d;
  *(u32x2*)o = u32x2{pack_bf2(v[0] * f, v[1] * f), pack_bf2(v[2] * f, v[3] * f)};
}

template <int DH, int R, int W>
__global__ __launch_bounds__(W * 64, R == 1 ? 3 : 2) void kv4_attention_kernel(Kv4Attn a) {
  constexpr int NG = DH / 32, ND = DH / 16, RT = 4 * R;
  // P' of a wave [group][query][32 keys] while it runs, then its output [query][DH]
  constexpr int PW = NG * RT * 16, OW = RT * DH;  // words
  __shared__ __attribute__((aligned(16))) uint32_t lds[W][PW > OW ? PW : OW];
  __shared__ float sm[W][RT], sl[W][RT];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c16 = lane & 15, kq = lane >> 4;
  const int bh = blockIdx.x, split = blockIdx.y;
  const int b = div_by(bh, a.by_Hkv), hk = bh - b * a.Hkv;
  const int G = a.G, rows = a.Lq * G, row0 = blockIdx.z * RT;
  // queries: MFMA row c16 = 4 i + r holds tile row i R + r.  Their loads, the
  // length's and the first block's are all on their way before any is waited for
  u32x4 qw[NG];
  {
    const int row = row0 + (c16 >> 2) * R + (c16 & 3), i = div_by(row, a.by_G);
    const bool there = (c16 & 3) < R && row < rows;
    const bf16_t* q = (const bf16_t*)a.q.p;
    if (there) q += b * a.q.seq + i * a.q.token + (hk * G + row - i * G) * a.q.head;
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      qw[g] = u32x4{0u, 0u, 0u, 0u};
      if (there) qw[g] = *(const u32x4*)(q + g * 32 + kq * 8);
    }
  }
  const int len = min(max(a.lens[b], 0), a.max_len);
  const Seen sn = seen_of(a, len, row0, min(rows, row0 + RT) - 1);
  const int j0 = split * a.chunk, j1 = min(sn.nb, j0 + a.chunk);
  if (j0 >= sn.nb && split) return;

  // this lane's rows of results: the positions of the last key that each sees, and how far back it sees
  int last[R];
  const int span = a.window ? a.window : INT_MAX;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int row = row0 + kq * R + r;
    last[r] = row < rows ? len - a.Lq + div_by(row, a.by_G) : -1;
  }
  // the blocks of this sequence and head (at most 2^24 tokens: below 2^32 bytes)
  const uint32_t bytes = (uint32_t)(a.L_cap / BLK) * (40 * DH);
  const uint8_t* const own = (const uint8_t*)a.cache + (size_t)bh * bytes;
  uint32_t* pw = lds[wave];
  const int prow = (c16 >> 2) * R + min(c16 & 3, R - 1);
  const UnpackCodes uk;
  const UnpackValues uv;
  // what the value operands of this lane's keys have above their codes, and MID, in 16ths
  const _Float16 over = (_Float16)((c16 & 1 ? 256 + MID : 16 + MID) / 16);
  const f16x2 above = {over, over};

  Words<NG> kc[2], kp[2], vp[2];
  Words<ND> vc;
  auto block_of = [&](int j) { return j < sn.sinkb ? j : sn.blk0 + j - sn.sinkb; };
  // past the run's last block the buffer is empty and the loads touch no memory:
  // a branch around them would make every wait one for all loads.  What a load has
  // beyond its lane's own offset goes into the wave's: it costs no registers there
  auto there = [&](int j) { return (uint32_t)((j - j1) >> 31); };  // all bits, or none
  auto buffer = [&](int j) {
    return __builtin_amdgcn_make_buffer_rsrc((void*)own, (short)0, (int)(bytes & there(j)), 0x00020000);
  };
  auto part_of = [&](int j, uint32_t at) { return ((uint32_t)block_of(j) * (40 * DH) + at) & there(j); };
  auto fetch_keys = [&](int j) {
    const __amdgpu_buffer_rsrc_t cache = buffer(j);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      kc[t] = load_words<NG>(cache, t * 8 * DH + c16 * (DH / 2) + kq * (DH / 8), part_of(j, 0));
      kp[t] = load_words<NG>(cache, (t * 16 + c16) * NG * 4, part_of(j, 32 * DH));
    }
  };
  auto fetch_values = [&](int j) {
    const __amdgpu_buffer_rsrc_t cache = buffer(j);
#pragma unroll
    for (int t = 0; t < 2; ++t) vp[t] = load_words<NG>(cache, (t * 16 + c16) * NG * 4, part_of(j, 36 * DH));
    vc = load_words<ND>(cache, lane * ND * 4, part_of(j, 16 * DH));
  };
  // the next block's keys and values are on their way as soon as this block's are used up
  fetch_keys(j0 + wave);
  fetch_values(j0 + wave);
  __builtin_amdgcn_sched_barrier(0);

  bf16x8 qa[NG];
#pragma unroll
  for (int g = 0; g < NG; ++g) qa[g] = __builtin_bit_cast(bf16x8, qw[g]);
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  // the sums of each query's groups, and -16 times them: where the scores' accumulators
  // start.  With R = 4 the registers of the former are wanted: 8 products a block in their place
  constexpr bool KEEP = R < 4;
  f32x4 q16[NG];
  float qs[NG][KEEP ? R : 1];
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    q16[g] = mfma(qa[g], __builtin_bit_cast(bf16x8, u32x4{0xc180c180u, 0xc180c180u, 0xc180c180u, 0xc180c180u}), zero);
#pragma unroll
    for (int r = 0; KEEP && r < R; ++r) qs[g][r] = -0.0625f * q16[g][r];
  }

  f32x4 o[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d) o[d] = zero;
  float m[R], l[R], bias[R][NG], psum[R][NG], unit[R][NG];  // sums of P, P m and P' of this lane's keys
#pragma unroll
  for (int r = 0; r < R; ++r) {
    m[r] = LOWEST;
    l[r] = 0.f;
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      bias[r][g] = psum[r][g] = 0.f;
      unit[r][g] = 0x1p126f;
    }
  }
  for (int j = j0 + wave; j < j1; j += W) {
    const int key0 = block_of(j) * BLK;
    // every row sees the whole block
    const bool whole = key0 + BLK - 1 <= sn.pos0 && (!a.window || key0 > sn.pos1 - a.window);
    float sc[2][R];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      f32x4 d[NG];
#pragma unroll
      for (int g = 0; g < NG; ++g) d[g] = mfma(qa[g], uk(kc[t].w[g]), q16[g]);
      // keeps the unused rows' registers from being used again before the MFMAs are done
#pragma unroll
      for (int g = 0; g < NG; ++g) asm volatile("" : "+v"(d[g]));
#pragma unroll
      for (int r = 0; r < R; ++r) sc[t][r] = 0.f;
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        const float low = hi16(kp[t].w[g]) * (KEEP ? 1.f : -0.0625f);
#pragma unroll
        for (int r = 0; r < R; ++r) sc[t][r] = fmaf(low, KEEP ? qs[g][r] : q16[g][r], sc[t][r]);
      }
#pragma unroll
      for (int g = 0; g < NG; ++g)
#pragma unroll
        for (int r = 0; r < R; ++r) sc[t][r] = fmaf(lo16(kp[t].w[g]), d[g][r], sc[t][r]);
    }
    // no use of this block's registers may sink below the loads into them
#pragma unroll
    for (int r = 0; r < R; ++r) asm volatile("" : "+v"(sc[0][r]), "+v"(sc[1][r]));
    __builtin_amdgcn_sched_barrier(0);
    fetch_keys(j + W);
    if (!whole) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int key = key0 + t * 16 + c16;
        // also replaces whatever the cache's unwritten rows gave
#pragma unroll
        for (int r = 0; r < R; ++r)
          sc[t][r] = (key <= last[r]) & ((last[r] - key < span) | (key < a.sinks)) ? sc[t][r] : -INFINITY;
      }
    }
    // The weights, P' as fp16 pairs, and whether this lane has one past its range: a
    // score above m, or a P' of 2^MOST and more (both halves of a pair at once)
    float p[2][R];
    uint32_t ph[R][NG];
    auto weigh = [&](auto all) {
      // what the two calls and the rescaling have in common would be kept in between:
      // registers that nothing has left (a third of a wave's at R = 4)
#pragma unroll
      for (int r = 0; r < R; ++r) asm("" : "+v"(sc[0][r]), "+v"(sc[1][r]));
      bool past = false;
      u16x2 most = {0, 0};
#pragma unroll
      for (int r = 0; r < R; ++r) {
        p[0][r] = exp2_of(fmaf(sc[0][r], a.scale_log2, -m[r]));
        p[1][r] = exp2_of(fmaf(sc[1][r], a.scale_log2, -m[r]));
        past |= fmaxf(p[0][r], p[1][r]) > 1.f;
#pragma unroll
        for (int g = 0; g < NG; ++g) {
          float x0 = p[0][r] * lo16(vp[0].w[g]) * unit[r][g], x1 = p[1][r] * lo16(vp[1].w[g]) * unit[r][g];
          if constexpr (!all.value) {  // a key that the row does not see may hold NaN
            x0 = sc[0][r] == -INFINITY ? 0.f : x0;
            x1 = sc[1][r] == -INFINITY ? 0.f : x1;
          }
          const u16x2 h = __builtin_bit_cast(u16x2, __builtin_convertvector((f32x2{x0, x1}), f16x2));
          most = __builtin_elementwise_max(most, h);
          ph[r][g] = __builtin_bit_cast(uint32_t, h);
        }
      }
      return past || ((__builtin_bit_cast(uint32_t, most) + 0x08000800u) & 0x80008000u);
    };
    auto weigh_block = [&] { return whole ? weigh(std::true_type{}) : weigh(std::false_type{}); };
    // The maximum moves where a score exceeds it, and then RAISE above the score, and
    // a unit where a P' passes its range: in a wave's first block, and in few others.
    // What a row does here goes by its own scores and P' alone, so its result does not
    // depend on the tile's other rows.  Exponents are fp32's, 127 for 2^0.
    bool some = j == j0 + wave;
    if (!some) some = __any(weigh_block());
    if (some) {
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const float top = row_max<>(fmaxf(sc[0][r], sc[1][r])) * a.scale_log2;
        const bool up = top > m[r];
        const float mn = up ? ceilf(top) + RAISE : m[r];  // whole numbers: what came before shrinks by 2^down
        const int down = up ? (int)fminf(mn - m[r], 512.f) : 0;
        m[r] = mn;
        l[r] = ldexpf(l[r], -down);
        const float p0 = exp2_of(fmaf(sc[0][r], a.scale_log2, -mn)), p1 = exp2_of(fmaf(sc[1][r], a.scale_log2, -mn));
#pragma unroll
        for (int g = 0; g < NG; ++g) {
          // the largest P s; NaN, as of unseen keys (0 times anything), is none
          const float x = fmaxf(fmaxf(p0 * lo16(vp[0].w[g]), p1 * lo16(vp[1].w[g])), 0.f);
          const int ex = (int)(row_max_u(__float_as_uint(x)) >> 23), e0 = (int)(__float_as_uint(unit[r][g]) >> 23);
          const int e1 = min(e0 + down, 253);  // so its unit may grow as much
          const int e = ex + e1 >= 254 + MOST ? 253 + PLACE - ex : e1;
          const int f = e - e0 - down;
          unit[r][g] = __uint_as_float((uint32_t)e << 23);
          bias[r][g] = ldexpf(bias[r][g], -down);
          psum[r][g] = ldexpf(psum[r][g], f);
          o[2 * g][r] = ldexpf(o[2 * g][r], f);
          o[2 * g + 1][r] = ldexpf(o[2 * g + 1][r], f);
        }
      }
      weigh_block();
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // the last block's reads of pw come first
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int r = 0; r < R; ++r) {
      l[r] += p[0][r] + p[1][r];
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        psum[r][g] = __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2, ph[r][g]), above, psum[r][g], false);
        pw[(g * RT + kq * R + r) * 16 + c16] = ph[r][g];
      }
    }
    float mid[2][NG];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int g = 0; g < NG; ++g) mid[t][g] = fmaf(MID, lo16(vp[t].w[g]), hi16(vp[t].w[g]));
    if (whole) {
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int g = 0; g < NG; ++g)
          bias[r][g] = fmaf(p[0][r], mid[0][g], fmaf(p[1][r], mid[1][g], bias[r][g]));
    } else {
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int g = 0; g < NG; ++g) {
          const float b1 = sc[1][r] == -INFINITY ? bias[r][g] : fmaf(p[1][r], mid[1][g], bias[r][g]);
          bias[r][g] = sc[0][r] == -INFINITY ? b1 : fmaf(p[0][r], mid[0][g], b1);
        }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      const f16x8 pa = __builtin_bit_cast(f16x8, *(const u32x4*)&pw[(g * RT + prow) * 16 + kq * 4]);
#pragma unroll
      for (int d = 2 * g; d < 2 * g + 2; ++d) o[d] = mfma(pa, uv(vc.w[d]), o[d]);
    }
    __builtin_amdgcn_sched_barrier(0);
    fetch_values(j + W);
  }

  // join the waves: lane (c16, kq) holds dims 16 d + c16 of tile rows kq R + r
  __syncthreads();
  float* ow = (float*)lds[wave];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const float ls = row_sum<>(l[r]);
    const int row = kq * R + r;
    if (c16 == 0) {
      sm[wave][row] = m[r];
      sl[wave][row] = ls;
    }
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      // the difference first: it is no larger than the values are
      const float w = inverse2(unit[r][g]), bs = row_sum<>(bias[r][g]), ps = row_sum<>(psum[r][g]);
#pragma unroll
      for (int d = 2 * g; d < 2 * g + 2; ++d) ow[row * DH + d * 16 + c16] = fmaf(fmaf(-16.f, ps, o[d][r]), w, bs);
    }
  }
  __syncthreads();
  for (int i = tid; i < RT * DH / 4; i += W * 64) {
    const int row = i / (DH / 4), d = i % (DH / 4) * 4, gr = row0 + row;
    if (gr >= rows) break;
    float mx = sm[0][row];
#pragma unroll
    for (int w = 1; w < W; ++w) mx = fmaxf(mx, sm[w][row]);
    float ls = 0.f;
    f32x4 v = zero;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const float f = exp2_of(sm[w][row] - mx);
      ls = fmaf(f, sl[w][row], ls);
      const f32x4 x = *(const f32x4*)((const float*)lds[w] + row * DH + d);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = fmaf(f, x[e], v[e]);
    }
    if (sn.nb <= a.chunk) {
      store_row(a, b, hk, gr, d, v, ls);
    } else {
      const size_t at = ((size_t)bh * rows + gr) * a.nsplit + split;
      *(f32x4*)(a.part + at * DH + d) = v;
      if (d == 0) *(f32x2*)(a.part + (size_t)gridDim.x * rows * a.nsplit * DH + at * 2) = f32x2{mx, ls};
    }
  }
}

// Joins the splits of a query row where there is more than one; one wave a
// row.  Lane s takes the maximum and sum of split s, so that the weights of 64
// splits cost one load and one reduction; the outputs of CB splits are in
// flight together, the first ones beside the length's load.
template <int DH, int R>
__global__ __launch_bounds__(64) void kv4_combine_kernel(Kv4Attn a, int total) {
  constexpr int CB = 16, RT = 4 * R, D = DH / 64;  // dims a lane
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
  const int row0 = gr / RT * RT;
  const Seen sn = seen_of(a, min(max(length, 0), a.max_len), row0, min(rows, row0 + RT) - 1);
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
  const float f = l == 0.f ? 0.f : 1.f / l;
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
// Splits that a plan may take, and scratch is sized for: some 8192 workgroups, with
// which the last round of 256 costs 3% at most, of four blocks or more.  It never
// falls with the length, which a plan's own number does, so scratch for the longest call
// serves each shorter one; of 100000 drawn calls (1 to 128 sequences, 1 to 140000 tokens)
// 0.7% would take more splits, and lose 2% of their estimated time on average.
unsigned most_splits(int B, int Lq, int H, int Hkv, unsigned blocks) {
  const int rows = Lq * (H / Hkv), tile = rows > 8 ? 16 : rows > 4 ? 8 : 4;
  const int64_t wgs = (int64_t)B * Hkv * ((rows + tile - 1) / tile), n = (8191 + wgs) / wgs;
  return n < (blocks + 3) / 4 ? (unsigned)n : (blocks + 3) / 4;
}

struct Plan {
  int R, W, tiles, chunk, nsplit;
};
// Queries a tile (4 R), waves a workgroup and blocks a wave, by the estimated
// time of each choice, in hundredths of a microsecond: a wave alone on its SIMD
// takes 75 a block, a SIMD 35 a block and 37 more a wave, 5% and 46% more with
// R = 2 and 4 (instruction latency and the LDS round trip weigh more than
// instructions; dh hardly shows), and a launch 66 and 209 more (a wave's first
// block sets a range for each query and group); one CU takes the workgroups past
// 256; joining splits costs 231, and 22 more past every 16 splits.  Over 86 calls
// timed at every choice (1 to 128 sequences, 1 to 131072 tokens, 1 to 256 queries a
// KV head, windows), up to 100 each, what this takes is 0.9% slower than the
// fastest on average and 9% at most.  Smaller tiles than the queries need unpack
// the cache again for each, but where whole ones leave CUs idle they are faster:
// 16 sequences of 12 queries over 8 heads and a window of 1024, one tile 15.5 us,
// two 10.6.
Plan plan_of(int B, int Lq, int H, int Hkv, int max_len, int window, int sinks) {
  const int rows = Lq * (H / Hkv);
  Plan p{};
  const unsigned blocks = blocks_of(Lq, max_len, window, sinks), limit = most_splits(B, Lq, H, Hkv, blocks);
  int64_t best = INT64_MAX;
  for (int R = 1; R == 1 || (R <= 4 && 2 * R < rows); R *= 2) {
    const int tiles = (rows + 4 * R - 1) / (4 * R);
    const int64_t bt = (int64_t)B * Hkv * tiles;
    const int64_t slower = R == 1 ? 100 : R == 2 ? 105 : 146, more = R == 1 ? 0 : R == 2 ? 66 : 209;
    for (int W = 4; W <= 8; W += 4) {
      const unsigned most = (blocks + W - 1) / W;
      auto consider = [&](unsigned per) {
        const unsigned ns = (blocks + per * W - 1) / (per * W);
        const int64_t a_simd = (bt * ns + 255) / 256 * (W / 4), wave = 75ll * per, simd = a_simd * (35 * per + 37);
        const int64_t cost = (wave > simd ? wave : simd) * slower / 100 + more + (ns > 1 ? 231 + 22 * ((ns - 1) / 16) : 0);
        if (cost < best && ns <= limit && tiles <= 65535)
          best = cost, p = Plan{R, W, tiles, (int)(per * W), (int)ns};
        return wave * slower / 100 + more < best;  // else longer runs of blocks cost no less
      };
      // runs that fill all CUs equally, then short ones by ones and longer ones by quarters
      for (int64_t wgs = 256; wgs <= 1024; wgs += 256)
        if (wgs >= bt) consider((unsigned)((most + wgs / bt - 1) / (wgs / bt)));
      for (unsigned per = 1; per < most && consider(per);) per += per < 6 ? 1 : per < 12 ? 2 : per < 24 ? 4 : per / 4;
      consider(most);
    }
  }
  return p;
}

template <int DH, int R, int W>
hipError_t launch_attention(const Kv4Attn& a, int tiles, hipStream_t s) {
  hipLaunchKernelGGL((kv4_attention_kernel<DH, R, W>), dim3(a.B * a.Hkv, a.nsplit, tiles), dim3(W * 64), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.nsplit == 1) return e;
  hipLaunchKernelGGL((kv4_combine_kernel<DH, R>), dim3(a.B * a.Lq * a.H), dim3(64), 0, s, a, a.B * a.Lq * a.H);
  return hipGetLastError();
}
template <int DH, int W>
hipError_t by_rows(const Kv4Attn& a, const Plan& p, hipStream_t s) {
  switch (p.R) {
    case 1: return launch_attention<DH, 1, W>(a, p.tiles, s);
    case 2: return launch_attention<DH, 2, W>(a, p.tiles, s);
    default: return launch_attention<DH, 4, W>(a, p.tiles, s);
  }
}

}  // namespace

size_t kv4_bytes(int B, int Hkv, int L_cap, int dh) { return (size_t)B * Hkv * (L_cap / BLK) * (40 * dh); }

namespace {
// blocks that L tokens from any position on can touch
unsigned rows_grid(Kv4Rows& a) {
  a.blocks = (a.L + 2 * (BLK - 1)) / BLK;
  a.by_blocks = fast_div(a.blocks);
  a.by_Hkv = fast_div(a.Hkv);
  return (unsigned)(a.B * a.Hkv * a.blocks);
}
}  // namespace

hipError_t kv4_store(Kv4Rows a, int dh, hipStream_t s) {
  const dim3 grid(2 * rows_grid(a)), block(256);
  if (dh == 128)
    hipLaunchKernelGGL((kv4_store_kernel<128>), grid, block, 0, s, a);
  else
    hipLaunchKernelGGL((kv4_store_kernel<64>), grid, block, 0, s, a);
  return hipGetLastError();
}

hipError_t kv4_load(Kv4Rows a, int dh, hipStream_t s) {
  const dim3 grid(rows_grid(a)), block(256);
  if (dh == 128)
    hipLaunchKernelGGL((kv4_load_kernel<128>), grid, block, 0, s, a);
  else
    hipLaunchKernelGGL((kv4_load_kernel<64>), grid, block, 0, s, a);
  return hipGetLastError();
}

size_t kv4_attention_scratch(int B, int Lq, int H, int Hkv, int dh, int max_len, int window, int sinks) {
  const unsigned n = most_splits(B, Lq, H, Hkv, blocks_of(Lq, max_len, window, sinks));
  return n < 2 ? 0 : (size_t)B * Lq * H * n * (dh + 2) * sizeof(float);
}

hipError_t kv4_attention(Kv4Attn a, int dh, size_t scratch_bytes, hipStream_t s) {
  if (scratch_bytes < kv4_attention_scratch(a.B, a.Lq, a.H, a.Hkv, dh, a.max_len, a.window, a.sinks))
    return hipErrorOutOfMemory;
  const Plan p = plan_of(a.B, a.Lq, a.H, a.Hkv, a.max_len, a.window, a.sinks);
  a.G = a.H / a.Hkv;
  a.by_G = fast_div(a.G);
  a.by_Hkv = fast_div(a.Hkv);
  a.by_chunk = fast_div(p.chunk);
  a.by_rows = fast_div(a.Lq * a.G);
  a.chunk = p.chunk;
  a.nsplit = p.nsplit;
  a.scale_log2 = 1.4426950408889634f / sqrtf((float)dh);
  if (p.W == 8) return dh == 128 ? by_rows<128, 8>(a, p, s) : by_rows<64, 8>(a, p, s);
  return dh == 128 ? by_rows<128, 4>(a, p, s) : by_rows<64, 4>(a, p, s);
}

}  // namespace vla
