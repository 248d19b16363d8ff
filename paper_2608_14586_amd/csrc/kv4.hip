// The KV cache in 4 bits: rows into it, rows out of it, and attention over it.
//
// Every 32 dims of a key or value row are one group of 16 levels: s =
// bf16((max - min) / 15), m = min (a bf16 number already), code = (x - m) / s
// to the nearest, ties to the even one; the row stands for m + s code.
//
// The cache of one sequence and KV head is a run of blocks of 32 tokens, 40 dh
// bytes each, everything that attention needs of them side by side:
//   key codes    [token 32][quarter 4][group dh/32] words: the 8 codes of dims
//                32 group + 8 quarter + j, code j in nibble j / 2 (even j) or
//                4 + j / 2 (odd j)
//   value codes  [quarter 4][d % 16][d / 16] words: the 8 codes of dim d of
//                tokens 4 quarter + i (nibble i, low half) and 16 + 4 quarter + i
//                (nibble 4 + i), i < 4
//   key params   [token 32][group] words: s in the low half, m in the high
//   value params [token 32][group] words
// In this order a wave's loads of keys and values are contiguous and every
// 32-bit word of codes is one lane's operand of an MFMA step.
#include "kernels.h"

namespace vla {
namespace {

constexpr int BLK = 32;  // tokens per block
constexpr uint32_t BIAS16 = 0x41804180u;  // bf16 16.0 twice
constexpr uint32_t CODE_BITS = 0x00780078u;

// 8 codes of a word as bf16 numbers 16 + c (the code in the top four mantissa
// bits of a bf16 with the exponent of 16)
__device__ __forceinline__ bf16x8 unpack8(uint32_t w) {
  const u32x4 v = {(w << 3 & CODE_BITS) | BIAS16, (w >> 1 & CODE_BITS) | BIAS16, (w >> 5 & CODE_BITS) | BIAS16,
                   (w >> 9 & CODE_BITS) | BIAS16};
  return __builtin_bit_cast(bf16x8, v);
}
__device__ __forceinline__ float lo16(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi16(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ f32x4 mfma(const bf16x8& a, const bf16x8& b, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// ------------------------------------------------------------ rows in and out

struct Group4 {
  uint32_t codes;   // of this lane's 8 dims
  uint32_t params;  // of the group
};
// Quantises the 8 dims of this lane; the 4 lanes of a group hold its 32 dims.
// Half of every number is used, so that max - min cannot overflow.  The
// quotient is corrected once by its remainder: x - m and s have at most 17
// and 8 significant bits, so a quotient that lies on a border between codes
// is exactly representable, and comes out exact.
__device__ __forceinline__ Group4 quantise(const u32x4& w) {
  float x[8];
  uint32_t mag = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[2 * e] = lo16(w[e]);
    x[2 * e + 1] = hi16(w[e]);
    mag = max(mag, max(w[e] & 0x7fffu, w[e] >> 16 & 0x7fffu));
  }
  float lo = x[0], hi = x[0];
#pragma unroll
  for (int e = 1; e < 8; ++e) {
    lo = fminf(lo, x[e]);
    hi = fmaxf(hi, x[e]);
  }
#pragma unroll
  for (int o = 1; o < 4; o <<= 1) {
    lo = fminf(lo, __shfl_xor(lo, o));
    hi = fmaxf(hi, __shfl_xor(hi, o));
    mag = max(mag, (uint32_t)__shfl_xor((int)mag, o));
  }
  if (mag >= 0x7f80u) return Group4{0u, 0x7fc07fc0u};  // a value that is not finite: the group reads as NaN
  const float half = 0.5f * hi - 0.5f * lo;
  const uint32_t m = __float_as_uint(lo) & 0xffff0000u;
  if (!(half >= 0x1p-100f)) return Group4{0u, m};
  const uint16_t sb = f2bf(half / 7.5f);
  const float hs = 0.5f * bf2f(sb), inv = 1.f / hs;
  uint32_t c = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float t = fmaf(0.5f, x[e], -0.5f * lo);
    float q = t * inv;
    q = fmaf(fmaf(-q, hs, t), inv, q);
    c |= (uint32_t)fminf(rintf(q), 15.f) << 4 * (e / 2 + (e & 1) * 4);
  }
  return Group4{c, m | sb};
}

// this workgroup's block of the cache and the tokens of the call in it:
// tokens [t0, t1) of the block are tokens from + (t - t0) of the sequence's rows
struct Span {
  int b, h, blk, t0, t1, from;
};
__device__ __forceinline__ Span span_of(const Kv4Rows& a) {
  Span s;
  const int nb = a.L / BLK + 2;
  const int i = blockIdx.x % nb, bh = blockIdx.x / nb;
  s.h = bh % a.Hkv;
  s.b = bh / a.Hkv;
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

template <int DH>
__global__ __launch_bounds__(256) void kv4_store_kernel(Kv4Rows a) {
  constexpr int LPR = DH / 8, RPP = 256 / LPR, NG = DH / 32, ND = DH / 16;  // lanes a row, rows a pass
  __shared__ uint32_t vs[BLK][LPR];
  const Span s = span_of(a);
  if (s.t0 >= s.t1) return;
  uint8_t* base = (uint8_t*)a.cache + (((size_t)s.b * a.Hkv + s.h) * (a.L_cap / BLK) + s.blk) * (40 * DH);
  const int tid = threadIdx.x, j = tid % LPR, g = j / 4, kq = j % 4;
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    const Heads& in = p ? a.v : a.k;
#pragma unroll
    for (int r = 0; r < BLK / RPP; ++r) {
      const int t = r * RPP + tid / LPR;
      if (t < s.t0 || t >= s.t1) continue;
      const bf16_t* row = (const bf16_t*)in.p + s.b * in.seq + (int64_t)(s.from + t - s.t0) * in.token + s.h * in.head;
      const Group4 q = quantise(*(const u32x4*)(row + j * 8));
      if (p)
        vs[t][j] = q.codes;
      else
        *(uint32_t*)(base + t * (DH / 2) + kq * (DH / 8) + g * 4) = q.codes;
      if (kq == 0) *(uint32_t*)(base + (p ? 36 : 32) * DH + (t * NG + g) * 4) = q.params;
    }
  }
  __syncthreads();
  uint32_t* vc = (uint32_t*)(base + 16 * DH);
  for (int i = tid; i < 4 * DH; i += 256) {
    const int d = i % ND * 16 + i / ND % 16, q4 = i / DH * 4;
    const int sh = 4 * (d % 8 / 2 + (d & 1) * 4);
    uint32_t w = 0, have = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int t = q4 + e % 4 + e / 4 * 16;
      if (t >= s.t0 && t < s.t1) {
        w |= (vs[t][d / 8] >> sh & 15u) << 4 * e;
        have |= 15u << 4 * e;
      }
    }
    if (have == 0) continue;
    if (have != 0xffffffffu) w |= vc[i] & ~have;  // tokens of other calls keep theirs
    vc[i] = w;
  }
}

template <int DH>
__global__ __launch_bounds__(256) void kv4_load_kernel(Kv4Rows a) {
  constexpr int LPR = DH / 8, RPP = 256 / LPR, NG = DH / 32, ND = DH / 16;
  __shared__ uint32_t vs[4 * DH];
  const Span s = span_of(a);
  if (s.t0 >= s.t1) return;
  const uint8_t* base = (const uint8_t*)a.cache + (((size_t)s.b * a.Hkv + s.h) * (a.L_cap / BLK) + s.blk) * (40 * DH);
  const int tid = threadIdx.x, j = tid % LPR, g = j / 4, kq = j % 4;
  for (int i = tid; i < 4 * DH; i += 256) vs[i] = ((const uint32_t*)(base + 16 * DH))[i];
  __syncthreads();
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    const Heads& out = p ? a.v : a.k;
#pragma unroll
    for (int r = 0; r < BLK / RPP; ++r) {
      const int t = r * RPP + tid / LPR;
      if (t < s.t0 || t >= s.t1) continue;
      const uint32_t prm = *(const uint32_t*)(base + (p ? 36 : 32) * DH + (t * NG + g) * 4);
      const float sc = lo16(prm), mn = hi16(prm);
      const uint32_t kw = p ? 0u : *(const uint32_t*)(base + t * (DH / 2) + kq * (DH / 8) + g * 4);
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        uint32_t c;
        if (p) {
          const int d = j * 8 + e, w = (t % 16 / 4) * DH + (d % 16) * ND + d / 16;
          c = vs[w] >> 4 * (t % 4 + t / 16 * 4) & 15u;
        } else {
          c = kw >> 4 * (e / 2 + (e & 1) * 4) & 15u;
        }
        x[e] = fmaf(sc, (float)c, mn);
      }
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
//  * scores: 16 + c as a bf16 is made of a code by a shift and an and-or, so
//      q . k = sum_g [ s_g sum (16 + c) q + (m_g - 16 s_g) sum q ]
//    over the groups g of 32 dims: one MFMA step a group (queries against 16
//    keys) and two multiply-adds in fp32; sum q is a constant of the loop.
//  * softmax: a running maximum and sum per query, in fp32, one pass.
//  * values: with P the weights and per group P' = P s_g as hi + lo bf16 pairs
//    (a 16-bit significand; one bf16 alone would double the error of a bf16
//    output, since it multiplies 16 + c),
//      sum P v = sum P' (16 + c) + sum P (m_g - 16 s_g)
//    the first sum by MFMA, the second in fp32 in the lane that holds P.
// The 4 R queries of a tile sit in the MFMA rows 4 i + r, r < R, so with up to
// four of them a lane holds one useful score a key and not four (R = 1).
// P crosses from score lanes (one key each) to operand lanes (8 keys of one
// query) through LDS, as 32-bit pairs of the keys t and t + 16: that pairing
// is why the value codes of those tokens share a word's halves.
// Work is split over the keys: waves of a workgroup take every W-th block of
// 32 keys, workgroups contiguous runs of them, joined in LDS and by
// kv4_combine_kernel.

template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), CTRL, 0xf, 0xf, true));
}
// over the 16 lanes of a row
__device__ __forceinline__ float row_max(float x) {
  x = fmaxf(x, dpp<0xB1>(x));
  x = fmaxf(x, dpp<0x4E>(x));
  x = fmaxf(x, dpp<0x141>(x));
  return fmaxf(x, dpp<0x140>(x));
}
__device__ __forceinline__ float row_sum(float x) {
  x += dpp<0xB1>(x);
  x += dpp<0x4E>(x);
  x += dpp<0x141>(x);
  return x + dpp<0x140>(x);
}

template <int N>
struct Words {
  uint32_t w[N];
};
template <int N>
__device__ __forceinline__ Words<N> load_words(const uint8_t* p) {
  Words<N> r;
  if constexpr (N % 4 == 0) {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      const u32x4 v = *(const u32x4*)(p + 16 * i);
#pragma unroll
      for (int e = 0; e < 4; ++e) r.w[4 * i + e] = v[e];
    }
  } else {
    const u32x2 v = *(const u32x2*)p;
    r.w[0] = v[0];
    r.w[1] = v[1];
  }
  return r;
}

template <int DH, int R, int W>
__global__ __launch_bounds__(W * 64) void kv4_attention_kernel(Kv4Attn a) {
  constexpr int NG = DH / 32, ND = DH / 16, RT = 4 * R;
  // P' of a wave [hi, lo][group][query][32 keys] while it runs, then its output [query][DH]
  constexpr int PW = 2 * NG * RT * 16, OW = RT * DH;  // words
  __shared__ __attribute__((aligned(16))) uint32_t lds[W][PW > OW ? PW : OW];
  __shared__ float sm[W][RT], sl[W][RT];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c16 = lane & 15, kq = lane >> 4;
  const int G = a.H / a.Hkv, rows = a.Lq * G, tiles = (rows + RT - 1) / RT;
  const int split = blockIdx.x % a.nsplit, rt = blockIdx.x / a.nsplit % tiles, bh = blockIdx.x / a.nsplit / tiles;
  const int hk = bh % a.Hkv, b = bh / a.Hkv;
  const int len = min(max(a.lens[b], 0), a.max_len);
  const int row0 = rt * RT;

  // this lane's rows of results: the positions of the first and last key that each sees in its window
  int last[R], first[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int row = row0 + kq * R + r;
    last[r] = row < rows ? len - a.Lq + row / G : -1;
    first[r] = a.window ? last[r] - a.window + 1 : 0;
  }
  // the blocks that any row of the tile sees: those of the first tokens, then the window's
  const int pos0 = len - a.Lq + row0 / G, pos1 = len - a.Lq + (min(rows, row0 + RT) - 1) / G;
  const int lo = a.window ? max(pos0 - a.window + 1, 0) : 0;
  const int blk0 = lo / BLK, sinkb = min((min(a.sinks, lo) + BLK - 1) / BLK, blk0);
  const int nb = pos1 < 0 ? 0 : sinkb + pos1 / BLK + 1 - blk0;
  const int j0 = (int)((int64_t)split * nb / a.nsplit), j1 = (int)((int64_t)(split + 1) * nb / a.nsplit);

  // queries: MFMA row c16 = 4 i + r holds tile row i R + r
  bf16x8 qa[NG];
  {
    const int row = row0 + (c16 >> 2) * R + (c16 & 3);
    const bool there = (c16 & 3) < R && row < rows;
    const bf16_t* q = (const bf16_t*)a.q.p;
    if (there) q += b * a.q.seq + row / G * a.q.token + (hk * G + row % G) * a.q.head;
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      u32x4 v = {0u, 0u, 0u, 0u};
      if (there) v = *(const u32x4*)(q + g * 32 + kq * 8);
      qa[g] = __builtin_bit_cast(bf16x8, v);
    }
  }
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  f32x4 qs[NG];  // sums of each query's groups
#pragma unroll
  for (int g = 0; g < NG; ++g)
    qs[g] = mfma(qa[g], __builtin_bit_cast(bf16x8, u32x4{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u}), zero);

  f32x4 o[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d) o[d] = zero;
  float m[R], l[R], bias[R][NG];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    m[r] = -INFINITY;
    l[r] = 0.f;
#pragma unroll
    for (int g = 0; g < NG; ++g) bias[r][g] = 0.f;
  }
  const uint8_t* cache = (const uint8_t*)a.cache + ((size_t)b * a.Hkv + hk) * (a.L_cap / BLK) * (40 * DH);
  uint32_t* pw = lds[wave];

  for (int j = j0 + wave; j < j1; j += W) {
    const int blk = j < sinkb ? j : blk0 + j - sinkb;
    const uint8_t* base = cache + (size_t)blk * (40 * DH);
    Words<NG> kc[2], kp[2], vp[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      kc[t] = load_words<NG>(base + t * 8 * DH + c16 * (DH / 2) + kq * (DH / 8));
      kp[t] = load_words<NG>(base + 32 * DH + (t * 16 + c16) * NG * 4);
    }
    const Words<ND> vc = load_words<ND>(base + 16 * DH + lane * ND * 4);
#pragma unroll
    for (int t = 0; t < 2; ++t) vp[t] = load_words<NG>(base + 36 * DH + (t * 16 + c16) * NG * 4);
    // every row sees the whole block
    const bool whole = blk * BLK + BLK - 1 <= pos0 && (!a.window || blk * BLK > pos1 - a.window);

    float p[2][R];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
#pragma unroll
      for (int r = 0; r < R; ++r) p[t][r] = 0.f;
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        const f32x4 d = mfma(qa[g], unpack8(kc[t].w[g]), zero);
        const float s = lo16(kp[t].w[g]), mm = fmaf(-16.f, s, hi16(kp[t].w[g]));
#pragma unroll
        for (int r = 0; r < R; ++r) p[t][r] = fmaf(s, d[r], fmaf(mm, qs[g][r], p[t][r]));
      }
      const int key = blk * BLK + t * 16 + c16;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        p[t][r] *= a.scale_log2;
        // also replaces whatever the cache's unwritten rows gave
        if (!whole && !(key <= last[r] && (key >= first[r] || key < a.sinks))) p[t][r] = -INFINITY;
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const float mn = fmaxf(m[r], row_max(fmaxf(p[0][r], p[1][r])));
      const float ms = mn == -INFINITY ? 0.f : mn;
      const float al = exp2f(m[r] - ms);
      m[r] = mn;
      p[0][r] = exp2f(p[0][r] - ms);
      p[1][r] = exp2f(p[1][r] - ms);
      l[r] = l[r] * al + (p[0][r] + p[1][r]);
#pragma unroll
      for (int g = 0; g < NG; ++g) bias[r][g] *= al;
#pragma unroll
      for (int d = 0; d < ND; ++d) o[d][r] *= al;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // the last block's reads of pw come first
#pragma unroll
    for (int g = 0; g < NG; ++g)
#pragma unroll
      for (int r = 0; r < R; ++r) {
        float ps[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const float s = lo16(vp[t].w[g]), mm = fmaf(-16.f, s, hi16(vp[t].w[g]));
          // a key that the row does not see may hold NaN
          const bool seen = whole || p[t][r] != 0.f;
          ps[t] = seen ? p[t][r] * s : 0.f;
          bias[r][g] = seen ? fmaf(p[t][r], mm, bias[r][g]) : bias[r][g];
        }
        const uint32_t hi = pack_bf2(ps[0], ps[1]);
        const uint32_t rest = pack_bf2(ps[0] - lo16(hi), ps[1] - hi16(hi));
        pw[(g * RT + kq * R + r) * 16 + c16] = hi;
        pw[((NG + g) * RT + kq * R + r) * 16 + c16] = rest;
      }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const int prow = (c16 >> 2) * R + min(c16 & 3, R - 1);
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      const bf16x8 ph = __builtin_bit_cast(bf16x8, *(const u32x4*)&pw[(g * RT + prow) * 16 + kq * 4]);
      const bf16x8 pl = __builtin_bit_cast(bf16x8, *(const u32x4*)&pw[((NG + g) * RT + prow) * 16 + kq * 4]);
#pragma unroll
      for (int d = 2 * g; d < 2 * g + 2; ++d) {
        const bf16x8 v = unpack8(vc.w[d]);
        o[d] = mfma(ph, v, o[d]);
        o[d] = mfma(pl, v, o[d]);
      }
    }
    __builtin_amdgcn_wave_barrier();
  }

  // join the waves: lane (c16, kq) holds dims 16 d + c16 of tile rows kq R + r
  __syncthreads();
  float* ow = (float*)lds[wave];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const float ls = row_sum(l[r]);
    const int row = kq * R + r;
    if (c16 == 0) {
      sm[wave][row] = m[r];
      sl[wave][row] = ls;
    }
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      const float bs = row_sum(bias[r][g]);
#pragma unroll
      for (int d = 2 * g; d < 2 * g + 2; ++d) ow[row * DH + d * 16 + c16] = o[d][r] + bs;
    }
  }
  __syncthreads();
  for (int i = tid; i < RT * DH; i += W * 64) {
    const int row = i / DH, d = i % DH;
    if (row0 + row >= rows) break;
    float mx = -INFINITY;
#pragma unroll
    for (int w = 0; w < W; ++w) mx = fmaxf(mx, sm[w][row]);
    float ls = 0.f, v = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const float f = sm[w][row] == -INFINITY ? 0.f : exp2f(sm[w][row] - mx);
      ls = fmaf(f, sl[w][row], ls);
      v = fmaf(f, ((const float*)lds[w])[i], v);
    }
    if (a.nsplit == 1) {
      const int gr = row0 + row;
      ((bf16_t*)a.o.p)[b * a.o.seq + gr / G * a.o.token + (hk * G + gr % G) * a.o.head + d] =
          f2bf(ls == 0.f ? 0.f : v / ls);
    } else {
      float* part = a.part + (((size_t)bh * rows + row0 + row) * a.nsplit + split) * (DH + 2);
      part[2 + d] = v;
      if (d == 0) {
        part[0] = mx;
        part[1] = ls;
      }
    }
  }
}

// joins the splits of one query row (blockIdx.x), one thread a dim
template <int DH>
__global__ __launch_bounds__(DH) void kv4_combine_kernel(Kv4Attn a) {
  const int G = a.H / a.Hkv, rows = a.Lq * G;
  const int gr = blockIdx.x % rows, bh = blockIdx.x / rows, hk = bh % a.Hkv, b = bh / a.Hkv, d = threadIdx.x;
  const float* part = a.part + (size_t)blockIdx.x * a.nsplit * (DH + 2);
  float mx = -INFINITY;
  for (int s = 0; s < a.nsplit; ++s) mx = fmaxf(mx, part[s * (DH + 2)]);
  float l = 0.f, v = 0.f;
  for (int s = 0; s < a.nsplit; ++s) {
    const float* p = part + s * (DH + 2);
    const float f = p[0] == -INFINITY ? 0.f : exp2f(p[0] - mx);
    l = fmaf(f, p[1], l);
    v = fmaf(f, p[2 + d], v);
  }
  ((bf16_t*)a.o.p)[b * a.o.seq + gr / G * a.o.token + (hk * G + gr % G) * a.o.head + d] = f2bf(l == 0.f ? 0.f : v / l);
}

constexpr int W_ATT = 4;

struct Plan {
  int R, tiles, nsplit;
};
// Splits over the keys: enough workgroups for two a CU, as long as every wave has a block of its own.
Plan plan_of(int B, int Lq, int H, int Hkv, int max_len, int window, int sinks) {
  const int rows = Lq * (H / Hkv);
  Plan p;
  p.R = rows <= 4 ? 1 : rows <= 8 ? 2 : 4;
  p.tiles = (rows + 4 * p.R - 1) / (4 * p.R);
  int64_t blocks = cdiv(max_len, BLK);
  if (window > 0) {
    const int64_t w = ((int64_t)window + Lq - 1 + BLK - 1) / BLK + 1 + cdiv(sinks, BLK);
    if (w < blocks) blocks = w;
  }
  const int64_t wgs = (int64_t)B * Hkv * p.tiles;
  int64_t ns = (512 + wgs - 1) / wgs;
  const int64_t most = (blocks + W_ATT - 1) / W_ATT;
  if (ns > most) ns = most;
  p.nsplit = ns < 1 ? 1 : (int)ns;
  return p;
}

template <int DH, int R>
hipError_t launch_attention(const Kv4Attn& a, int tiles, hipStream_t s) {
  const int64_t grid = (int64_t)a.B * a.Hkv * tiles * a.nsplit;
  if (grid > 0x7fffffff) return hipErrorInvalidValue;
  hipLaunchKernelGGL((kv4_attention_kernel<DH, R, W_ATT>), dim3((unsigned)grid), dim3(W_ATT * 64), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.nsplit == 1) return e;
  hipLaunchKernelGGL((kv4_combine_kernel<DH>), dim3((unsigned)(a.B * a.H * a.Lq)), dim3(DH), 0, s, a);
  return hipGetLastError();
}
template <int DH>
hipError_t by_rows(const Kv4Attn& a, const Plan& p, hipStream_t s) {
  switch (p.R) {
    case 1: return launch_attention<DH, 1>(a, p.tiles, s);
    case 2: return launch_attention<DH, 2>(a, p.tiles, s);
    default: return launch_attention<DH, 4>(a, p.tiles, s);
  }
}

}  // namespace

size_t kv4_bytes(int B, int Hkv, int L_cap, int dh) { return (size_t)B * Hkv * (L_cap / BLK) * (40 * dh); }

hipError_t kv4_store(const Kv4Rows& a, int dh, hipStream_t s) {
  const dim3 grid((unsigned)(a.B * a.Hkv * (a.L / BLK + 2))), block(256);
  if (dh == 128)
    hipLaunchKernelGGL((kv4_store_kernel<128>), grid, block, 0, s, a);
  else
    hipLaunchKernelGGL((kv4_store_kernel<64>), grid, block, 0, s, a);
  return hipGetLastError();
}

hipError_t kv4_load(const Kv4Rows& a, int dh, hipStream_t s) {
  const dim3 grid((unsigned)(a.B * a.Hkv * (a.L / BLK + 2))), block(256);
  if (dh == 128)
    hipLaunchKernelGGL((kv4_load_kernel<128>), grid, block, 0, s, a);
  else
    hipLaunchKernelGGL((kv4_load_kernel<64>), grid, block, 0, s, a);
  return hipGetLastError();
}

size_t kv4_attention_scratch(int B, int Lq, int H, int Hkv, int dh, int max_len, int window, int sinks) {
  const Plan p = plan_of(B, Lq, H, Hkv, max_len, window, sinks);
  return p.nsplit == 1 ? 0 : (size_t)B * Lq * H * p.nsplit * (dh + 2) * sizeof(float);
}

hipError_t kv4_attention(Kv4Attn a, int dh, hipStream_t s) {
  const Plan p = plan_of(a.B, a.Lq, a.H, a.Hkv, a.max_len, a.window, a.sinks);
  a.nsplit = p.nsplit;
  a.scale_log2 = 1.4426950408889634f / sqrtf((float)dh);
  return dh == 128 ? by_rows<128>(a, p, s) : by_rows<64>(a, p, s);
}

}  // namespace vla
