// Causal attention over packed prompts (bf16 MFMA, fp32 online softmax).
//
//   o_t = sum_{j <= t} exp(q_t k_j / sqrt(dh) - m_t) v_j / sum_{j <= t} exp(...)   within a prompt
//
// Bound by the matrix cores: 4 dh operations a pair of a query and a key that it sees.
// One workgroup of 4 waves takes 128 queries of a prompt and head, a wave 32 of them
// side by side.  Keys advance in tiles of 64 that all waves share, K and V as they
// lie in memory, rows of dh, moved by buffer_load ... lds into two stages; rows past the
// prompt's end read as zero through the buffer, whatever lies there.
//
// Scores are formed transposed, S^T = K Q^T (32x32x16), so that a lane holds 16 keys of
// one query: its maximum and sum need one exchange with the lane 32 away, and its
// weights are the operand of O^T = V^T P^T as they lie, for the keys 16 s + 4 h + j and 16 s
// + 8 + 4 h + j (h = lane / 32, j < 4) of each k-step.  V's operand, those keys of one dim,
// is read with a transposing LDS load (ds_read_b64_tr_b16: four keys of 16 dims a group
// of 16 lanes), so nothing is transposed beforehand.  Weights are rounded to bf16, since values are bf16
// and an MFMA's operands of one type: 2^-8 of each at most, and 0.0019 to 0.0020 of the result against 64 bits, where its
// own rounding alone gives 0.0016.  The sum is of the rounded weights, two a v_dot2, so both are rounded alike.
//
// A wave works one tile ahead: between the exponentials of tile t its MFMAs form the
// scores of tile t + 1.  One long prompt (16384 tokens, 8 heads of 128) takes 530 to 545 us, 1010 to
// 1040 TF/s of the half that is not masked, four prompts of 4096, 2048, 1201 and 847, 32 heads, 217 to 222: the matrix cores
// are busy for 52% and 42% of the cycles, at the 1.7 to 1.95 GHz that the chip holds under it.  Their operands, 1 KB from
// LDS for each MFMA of 32 cycles, take as long at 128 bytes a cycle (no bank conflicts), and so do exponentials and what else the
// softmax asks of the vector unit, by instruction counts; a SIMD's two waves overlap the three in part.  One prompt of
// 2048, 32 heads: 48 us (attention_bf16.hip, whose values come transposed, 43 to 45).  With less to do a tile takes a workgroup that has a CU alone 1.05 us, its
// parts one behind the other: without the loads 0.93, without exponentials 1.0, without
// three quarters of the PV products 1.0.  What did not help: 64 queries a wave (half the LDS reads,
// but 268 us for 225: accumulators wander between the register files), the next tile's maximum and
// half of its weights between the PV products (16384 tokens 4% faster, prompts of 2048 4%
// slower), a third stage of values (0 to 10% slower), and key tiles dealt out to two groups of four
// waves (10 to 18% faster where fewer than 256 workgroups have 15 tiles and more, else slower;
// and a prompt's bits would depend on the others of the call), nor 64 queries a workgroup with two waves
// on the halves of each key tile, for prompts of up to 1024 (14 heads of 64: one of 1024 16.5 -> 12.8 us,
// nine of 1 to 701 12.9 -> 12.2, but 64 of 512 77 -> 102).
//
// Only a wave's last tile has masked keys, in one half of its 64 (the other is seen by all of
// the wave's queries, or by none).  A value there that is not finite must not reach the
// queries that do not see it (0 NaN is NaN): such are looked for, and where there is one
// (rarely) they are taken as 0, and a product of (not finite) with (sees it) marks what they
// make NaN.
//
// Workgroups take tiles of queries longest first (found from the offsets by each one), all
// heads of a tile side by side.
#include <math.h>

#include <type_traits>

#include "kernels.h"
#include "packed_order.h"

namespace vla {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int BKV = 64;
// A maximum before any score: finite, and below every finite score, so that scores of -inf have the weight 0, also
// where a query has met no other.  A query that meets none at all has the sum 0, and NaN for a result.
constexpr float LOWEST = -3e38f;

// (the row is in the vector offset, which the buffer's range check is sure to count; the scalar one it need not)
__device__ __forceinline__ void dma16(__amdgpu_buffer_rsrc_t r, void* lds, unsigned voff) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)lds, 16, voff, 0, 0, 0);
}
// every load of this wave has landed, every LDS access is done; then all waves meet
__device__ __forceinline__ void landed() {
  __builtin_amdgcn_s_waitcnt(0x0070);
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// over the wave, without a trip through LDS for each step
template <int CTRL>
__device__ __forceinline__ int dpp_i(int x) {
  return __builtin_amdgcn_update_dpp(0, x, CTRL, 0xf, 0xf, true);
}
__device__ __forceinline__ int wave_sum_i(int v) {
  v += dpp_i<0xB1>(v);
  v += dpp_i<0x4E>(v);
  v += dpp_i<0x141>(v);
  v += dpp_i<0x140>(v);
  return __builtin_amdgcn_readlane(v, 0) + __builtin_amdgcn_readlane(v, 16) + __builtin_amdgcn_readlane(v, 32) +
         __builtin_amdgcn_readlane(v, 48);
}

// The tile of BQ queries and the head (of H, some order) of workgroup `wg`: prompt rows
// [start, start + len), queries from q0 on; len = 0 where there is no such tile.  Up to 64
// prompts, tiles come longest first, all heads of one side by side, in the order of packed_rank: tile
// number n of a prompt has n + 1 tiles' work, and F(n) = sum over prompts of max(tiles - n, 0) tiles have
// number n or more.  More prompts: one behind the other.
struct Work {
  int start, len, q0, head;
};
__device__ __forceinline__ Work work_of(const PackedAttn& p, int wg, int BQ) {
  const int32_t* offsets = p.offsets;
  const int n_seq = p.n_seq, T = p.T, H = p.H;
  const int lane = threadIdx.x & 63;
  auto lane_seq = [&](int from, int& start, int& len) {
    const int i = from + lane;
    const int a = i < n_seq ? offsets[i] : 0, b = i < n_seq ? offsets[i + 1] : 0;
    start = min(max(a, 0), T);
    len = max(min(max(b, 0), T) - start, 0);
    return (len + BQ - 1) / BQ;
  };
  Work w{0, 0, 0, 0};
  int start, len, nt, pick = -1, tile = 0, id;
  if (n_seq <= 64) {
    nt = lane_seq(0, start, len);
    // total * H: the launch has at least as many workgroups, below 2^24
    const int rank = packed_rank(wg, wave_sum_i(nt), H, [&](int n) { return div_by(n, p.by_H); });
    if (rank < 0) return w;
    id = div_by(rank, p.by_H);
    w.head = rank - id * H;
    int lo = 0, hi = (T + BQ - 1) / BQ, more = 0;  // F(lo) > id >= F(hi) = more
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2, f = wave_sum_i(max(nt - mid, 0));
      if (f > id)
        lo = mid;
      else
        hi = mid, more = f;
    }
    uint64_t has = __ballot(nt > lo);
    for (int k = id - more; k > 0; --k) has &= has - 1;
    pick = __builtin_ctzll(has);
    tile = lo;
  } else {
    id = div_by(wg, p.by_H);
    w.head = wg - id * H;
    int before = 0;
    for (int from = 0; from < n_seq; from += 64) {
      nt = lane_seq(from, start, len);
      int upto = nt;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int x = __shfl_up(upto, o, 64);
        if (lane >= o) upto += x;
      }
      const uint64_t past = __ballot(before + upto > id);
      if (past) {
        pick = __builtin_ctzll(past);
        tile = id - before - __shfl(upto - nt, pick, 64);
        break;
      }
      before += __shfl(upto, 63, 64);
    }
    if (pick < 0) return w;
  }
  w.start = __builtin_amdgcn_readfirstlane(__shfl(start, pick, 64));
  w.len = __builtin_amdgcn_readfirstlane(__shfl(len, pick, 64));
  w.q0 = __builtin_amdgcn_readfirstlane(tile) * BQ;
  return w;
}

template <int DH>
__global__ __launch_bounds__(256, DH == 128 ? 2 : 3) void attention_packed_kernel(PackedAttn a) {
  constexpr int ROWB = DH * 2, TILE = BKV * ROWB, LOADS = TILE / 1024 / 4;  // 1 KB loads a wave and tile of K or V
  constexpr int RPK = 1024 / ROWB, CPR = ROWB / 16;                         // rows a load, 16-byte chunks a row
  constexpr int ND = DH / 32, KS = DH / 16, BQ = 128;
  // one array per operand and stage: the compiler can tell reads from the loads into other arrays
  __shared__ __attribute__((aligned(1024))) char sk0[TILE];
  __shared__ __attribute__((aligned(1024))) char sk1[TILE];
  __shared__ __attribute__((aligned(1024))) char sv0[TILE];
  __shared__ __attribute__((aligned(1024))) char sv1[TILE];

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = lane >> 5, li = lane & 31;
  const Work wk = work_of(a, blockIdx.x, BQ);
  if (wk.len == 0) return;
  // 8 heads side by side go to the 8 XCDs, each with a KV head's own queries where there are 8 KV heads
  const int gi = div_by(wk.head, a.by_Hkv), hk = wk.head - gi * a.Hkv, h = hk * a.G + gi;
  const int L = wk.len, q0 = wk.q0, qw0 = q0 + wave * 32;

  const bf16_t* kh = (const bf16_t*)a.k.p + (int64_t)wk.start * a.k.token + hk * a.k.head;
  const bf16_t* vh = (const bf16_t*)a.v.p + (int64_t)wk.start * a.v.token + hk * a.v.head;

  // the wave's queries as MFMA B operands; lanes past L load row L - 1 (not stored)
  const int qi = qw0 + li;
  bf16x8 fq[KS];
  {
    const bf16_t* row = (const bf16_t*)a.q.p + (int64_t)(wk.start + min(qi, L - 1)) * a.q.token + h * a.q.head;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) fq[ks] = *(const bf16x8*)(row + ks * 16 + half * 8);
  }
  const int ntiles = (min(L, q0 + BQ) + BKV - 1) / BKV;
  const int full = qw0 / BKV;  // tiles that the wave's queries see whole; the next one is its last
  const bool work = qw0 < L;

  // K row r: chunk c stored at c ^ ksw(r), so that 32 rows of one chunk meet every bank alike; V row r: at c ^ vsw(r), so
  // that 4 rows of 4 chunks side by side do
  auto ksw = [](int r) { return DH == 128 ? (r & 15) : ((r >> 1) & 7); };
  auto vsw = [](int r) { return DH == 128 ? (r & 3) << 2 : ((r >> 1) & 1) << 2; };
  auto rows_at = [&](const bf16_t* p, int64_t token, int t) {
    const int n = min(L - t * BKV, BKV);
    return __builtin_amdgcn_make_buffer_rsrc((void*)(p + (int64_t)t * BKV * token), (short)0,
                                             n > 0 ? (int)((n - 1) * token * 2 + ROWB) : 0, 0x00020000);
  };
  unsigned kv[LOADS], vv;
  {
    const int r0 = wave * LOADS * RPK + lane / CPR, cs = lane % CPR;
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      const int r = r0 + j * RPK;
      kv[j] = (unsigned)(r * a.k.token * 2) + (cs ^ ksw(r)) * 16;
    }
    vv = (unsigned)(r0 * a.v.token * 2) + (cs ^ vsw(r0)) * 16;
    static_assert(DH != 64 || RPK % 4 == 0, "vsw is the same in every load of a lane");
    static_assert(DH != 128 || RPK % 4 == 0, "vsw is the same in every load of a lane");
  }
  auto issue_k = [&](char* st, int t) {
    const __amdgpu_buffer_rsrc_t r = rows_at(kh, a.k.token, t);
#pragma unroll
    for (int j = 0; j < LOADS; ++j) dma16(r, st + (wave * LOADS + j) * 1024, kv[j]);
  };
  auto issue_v = [&](char* st, int t) {
    const __amdgpu_buffer_rsrc_t r = rows_at(vh, a.v.token, t);
#pragma unroll
    for (int j = 0; j < LOADS; ++j) dma16(r, st + (wave * LOADS + j) * 1024, vv + (unsigned)(j * RPK * a.v.token * 2));
  };

  f32x16 acc[ND];
#pragma unroll
  for (int t = 0; t < ND; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[t][r] = 0.f;
  float m = LOWEST, l = 0.f;

  // K tile t + 2 and V tile t + 1 go out at the head of tile t, into the stages that tile t - 1 read last
  issue_k(sk0, 0);
  issue_k(sk1, 1);
  issue_v(sv0, 0);

  f32x16 sa[2], sb[2];  // scores of the tile in work and of the next
  const f32x16 zero = {};
  auto kfrag = [&](const char* st, int t, int ks) -> bf16x8 {
    const int r = t * 32 + li, c = ks * 2 + half;
    return *(const bf16x8*)(st + r * ROWB + ((c ^ ksw(r)) * 16));
  };
  // keys 16 c4 + 4 half + j (and 8 further), j < 4, of dim 32 dt + li: lane i of 16 gives the address of row i / 4's
  // dims 4 (i % 4) ..
  const int vrow = half * 4 + (lane & 15) / 4;
  const int vcol = (lane >> 4 & 1) * 16 + (lane & 3) * 4;
  auto vfrag = [&](char* st, int c4, int dt) -> bf16x8 {
    const int r = c4 * 16 + vrow, c = (dt * 32 + vcol) / 8;
    char* p = st + r * ROWB + ((c ^ vsw(r)) * 16) + (lane & 1) * 8;
    const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p);
    const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(p + 8 * ROWB));
    typedef short s16x8 __attribute__((ext_vector_type(8)));
    return __builtin_bit_cast(bf16x8, (s16x8)__builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
  };
  landed();
  if (work) {
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        sa[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kfrag(sk0, t, ks), fq[ks], ks == 0 ? zero : sa[t], 0, 0, 0);
      }
  }
  const bf16x2 ones = {(__bf16)1.f, (__bf16)1.f}, none = {(__bf16)0.f, (__bf16)0.f};

  // the running maximum moves where a score is 8 (in log2) above it
  auto raise = [&](const f32x16(&s)[2]) {
    float top = fmaxf(s[0][0], s[1][0]);
#pragma unroll
    for (int r = 1; r < 16; ++r) top = fmaxf(fmaxf(top, s[0][r]), s[1][r]);
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
    top = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])) * a.scale_log2;
    if (__any(top > m + 8.f)) {
      // by the query's own scores alone: its bits do not depend on its neighbours
      const float mn = top > m + 8.f ? top : m, f = __builtin_amdgcn_exp2f(m - mn);
      l *= f;
#pragma unroll
      for (int t = 0; t < ND; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[t][r] *= f;
      m = mn;
    }
  };
  // weights x, x + 1 (x = 16 t + r) as a bf16 pair, added to the sum
  auto weigh = [&](const f32x16(&s)[2], int x) {
    const float p0 = __builtin_amdgcn_exp2f(fmaf(s[x >> 4][x & 15], a.scale_log2, -m));
    const float p1 = __builtin_amdgcn_exp2f(fmaf(s[x >> 4][(x & 15) + 1], a.scale_log2, -m));
    const bf16x2 w = {(__bf16)p0, (__bf16)p1};
    l = __builtin_amdgcn_fdot2_f32_bf16(w, ones, l, false);
    return __builtin_bit_cast(uint32_t, w);
  };
  auto operand = [](const uint32_t* p) { return __builtin_bit_cast(bf16x8, u32x4{p[0], p[1], p[2], p[3]}); };

  // an operand with zeros for what is not finite, and ones there in *is
  auto without = [](bf16x8 f, bf16x8* is) {
    u32x4 w = __builtin_bit_cast(u32x4, f), one;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t hit = ((w[e] & 0x7f80u) == 0x7f80u ? 0xffffu : 0u) | ((w[e] & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u);
      one[e] = hit & 0x3f803f80u;
      w[e] &= ~hit;
    }
    if (is) *is = __builtin_bit_cast(bf16x8, one);
    return __builtin_bit_cast(bf16x8, w);
  };
  // outputs of the queries that see a value of half t of a last tile that is not finite become NaN
  auto mark = [&](f32x16(&o)[ND], char* vst, int t) {
#pragma unroll
    for (int dt = 0; dt < ND; ++dt) {
      f32x16 hits = zero;
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        u32x4 see;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int key = c * 16 + (e >> 1) * 8 + half * 4 + (e & 1) * 2;  // of the half
          see[e] = (key <= li ? 0x3f80u : 0u) | (key + 1 <= li ? 0x3f800000u : 0u);
        }
        bf16x8 is;
        without(vfrag(vst, 2 * t + c, dt), &is);
        hits = __builtin_amdgcn_mfma_f32_32x32x16_bf16(is, __builtin_bit_cast(bf16x8, see), hits, 0, 0, 0);
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) o[dt][r] = hits[r] > 0.f ? __uint_as_float(0x7fc00000u) : o[dt][r];
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  // tile it in stage S (= it % 2): s holds its scores, sn receives the next tile's
  auto body = [&](auto S_, int it, f32x16(&s)[2], f32x16(&sn)[2]) {
    constexpr int S = decltype(S_)::value;
    // K tile it + 1 and V tile it landed, and every wave is done with the stages that the next loads overwrite
    landed();
    char* vst = S == 0 ? sv0 : sv1;
    const char* kst = S == 0 ? sk1 : sk0;
    if (it + 1 < ntiles) {
      issue_k(S == 0 ? sk0 : sk1, it + 2);
      issue_v(S == 0 ? sv1 : sv0, it + 1);
    }
    if (work && it < full) {
      uint32_t p[16];
      // operands in order: the next tile's K (NK), then this tile's V; read LA ahead of the MFMAs that take them.
      // The scheduling barriers let only VALU and scalar instructions cross, so this order is the one issued.
      constexpr int NK = 2 * KS, NP = 4 * ND, LA = 4;
      bf16x8 fr[LA];
      auto fetch = [&](int i) {
        if (i < NK)
          fr[i % LA] = kfrag(kst, i & 1, i >> 1);
        else if (i < NK + NP)
          fr[i % LA] = vfrag(vst, (i - NK) / ND, (i - NK) % ND);
      };
#pragma unroll
      for (int i = 0; i < LA; ++i) fetch(i);
      __builtin_amdgcn_sched_barrier(0);
      raise(s);
#pragma unroll
      for (int i = 0; i < NK; ++i) {
        const int ks = i >> 1, t = i & 1;
        sn[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr[i % LA], fq[ks], ks == 0 ? zero : sn[t], 0, 0, 0);
        fetch(i + LA);
#pragma unroll
        for (int x = i * 16 / NK; x < (i + 1) * 16 / NK; ++x) p[x] = weigh(s, 2 * x);
        __builtin_amdgcn_sched_barrier(0x406);
      }
#pragma unroll
      for (int j = 0; j < NP; ++j) {
        acc[j % ND] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr[(NK + j) % LA], operand(p + 4 * (j / ND)), acc[j % ND], 0, 0, 0);
        fetch(NK + j + LA);
        __builtin_amdgcn_sched_barrier(0x406);
      }
    }
  };
  for (int base = 0; base < ntiles; base += 2) {
    body(std::integral_constant<int, 0>{}, base, sa, sb);
    if (base + 1 < ntiles) body(std::integral_constant<int, 1>{}, base + 1, sb, sa);
  }
  // The wave's last tile: of its two halves of 32 keys, `diag` up to the query's own, the one before it whole, none
  // after.  The last two tiles' values are both still there.
  if (!work) return;
  {
    char* const vst = full & 1 ? sv1 : sv0;
    if (full & 1) sa[0] = sb[0], sa[1] = sb[1];
    const int diag = wave & 1;
    uint32_t p[16];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int key = t * 32 + (r >> 2) * 8 + half * 4 + (r & 3);
        sa[t][r] = key <= diag * 32 + li ? sa[t][r] : -INFINITY;
      }
    raise(sa);
#pragma unroll
    for (int x = 0; x < 16; ++x) p[x] = weigh(sa, 2 * x);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      if (t > diag) break;
      __builtin_amdgcn_sched_barrier(0);
      bool dirty = false;
      if (t == diag) {
        float bad = 0.f;
#pragma unroll
        for (int i = 0; i < 2 * ND; ++i) {
          const u32x4 w = __builtin_bit_cast(u32x4, vfrag(vst, 2 * t + i / ND, i % ND));
#pragma unroll
          for (int e = 0; e < 4; ++e)
            bad = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, (uint32_t)w[e]), none, bad, false);
          if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);
        }
        dirty = __any(bad != bad);
        if (dirty) mark(acc, vst, t);
      }
#pragma unroll
      for (int i = 0; i < 2 * ND; ++i) {
        bf16x8 f = vfrag(vst, 2 * t + i / ND, i % ND);
        if (dirty) f = without(f, nullptr);
        acc[i % ND] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, operand(p + 4 * (2 * t + i / ND)), acc[i % ND], 0, 0, 0);
        if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);
      }
    }
  }

  const float total = l + __shfl_xor(l, 32, 64);
  if (qi < L) {
    const float inv = 1.f / total;
    bf16_t* row = (bf16_t*)a.o.p + (int64_t)(wk.start + qi) * a.o.token + h * a.o.head;
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *(u32x2*)(row + dt * 32 + g * 8 + half * 4) =
            u32x2{pack_bf2(acc[dt][g * 4 + 0] * inv, acc[dt][g * 4 + 1] * inv),
                  pack_bf2(acc[dt][g * 4 + 2] * inv, acc[dt][g * 4 + 3] * inv)};
  }
}

template <int DH>
hipError_t launch(const PackedAttn& a, hipStream_t s) {
  // every tile but a prompt's last has 128 queries
  const int64_t wgs = ((int64_t)a.T / 128 + a.n_seq) * a.H;
  if (wgs >= 1ll << 24) return hipErrorInvalidValue;  // fewer than 2^32 threads
  hipLaunchKernelGGL((attention_packed_kernel<DH>), dim3((unsigned)wgs), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t attention_packed(PackedAttn a, int dh, hipStream_t s) {
  a.G = a.H / a.Hkv;
  a.by_H = fast_div(a.H);
  a.by_Hkv = fast_div(a.Hkv);
  a.scale_log2 = 1.4426950408889634f / sqrtf((float)dh);
  return dh == 128 ? launch<128>(a, s) : launch<64>(a, s);
}

}  // namespace vla
