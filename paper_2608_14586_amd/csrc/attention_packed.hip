// Causal attention over packed prompts (bf16 MFMA, fp32 online softmax).
//
//   o_t = sum_{j <= t} exp(q_t k_j / sqrt(dh) - m_t) v_j / sum_{j <= t} exp(...)   within a prompt
//
// Bound by the matrix cores: 4 dh operations a pair of a query and a key that it sees.
// One workgroup of 4 waves takes 128 NQ queries of a prompt and head, a wave 32 NQ of
// them side by side.  Keys advance in tiles of 64 that all waves share, K and V as they
// lie in memory, rows of dh, moved by buffer_load ... lds into two stages; rows past the
// prompt's end read as zero through the buffer, whatever lies there.
//
// Scores are formed transposed, S^T = K Q^T (32x32x16), so that a lane holds 16 keys of
// one query: its maximum and sum need one exchange with the lane 32 away, and its
// weights are the operand of O^T = V^T P^T as they lie, for the keys 16 s + 4 h + j and 16 s
// + 8 + 4 h + j (h = lane / 32, j < 4) of each k-step.  V's operand, those keys of one dim,
// is read with a transposing LDS load (ds_read_b64_tr_b16: four keys of 16 dims a group
// of 16 lanes), so nothing is transposed beforehand.  The sum is of the rounded weights,
// two a v_dot2, so weights and sum are rounded alike.
//
// A wave works one tile ahead: between the exponentials of tile t its MFMAs form the
// scores of tile t + 1.  With NQ = 2 every operand that is read from LDS serves two
// MFMAs.  At NQ = 1 LDS, 128 bytes a cycle, is as busy as the matrix cores: 1 KB a
// 32-cycle MFMA on each of 4 SIMDs.
//
// Only a wave's last tile has masked keys, and there only one half of 32 keys a set of 32
// queries.  A value there that is not finite must not reach the queries that do not see it
// (0 NaN is NaN): they are looked for, and where there is one (rarely) such values are
// taken as 0 and a product of (not finite) with (sees it) marks what they make NaN.
//
// Workgroups take tiles of queries longest first (found from the offsets by each one), all
// heads of a tile side by side.
#include <math.h>

#include <type_traits>

#include "kernels.h"

namespace vla {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int BKV = 64;

__device__ __forceinline__ void dma16(__amdgpu_buffer_rsrc_t r, void* lds, unsigned voff, int soff) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)lds, 16, voff, soff, 0, 0);
}
// every load of this wave has landed, every LDS access is done; then all waves meet
__device__ __forceinline__ void landed() {
  __builtin_amdgcn_s_waitcnt(0x0070);
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

__device__ __forceinline__ int wave_sum_i(int v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return __builtin_amdgcn_readfirstlane(v);
}

// Tile number `id` of the call's, in tiles of BQ queries: prompt rows [start, start +
// len), queries from q0 on; len = 0 where there is no such tile.  Up to 64 prompts, tiles
// come in the order of their lengths: tile number n of a prompt has n + 1 tiles' work, and
// F(n) = sum over prompts of max(tiles - n, 0) tiles have number n or more.  More prompts:
// one behind the other.
struct Work {
  int start, len, q0;
};
__device__ __forceinline__ Work work_of(const int32_t* offsets, int n_seq, int T, int id, int BQ) {
  const int lane = threadIdx.x & 63;
  auto lane_seq = [&](int first, int& start, int& len) {
    const int i = first + lane;
    const int a = i < n_seq ? offsets[i] : 0, b = i < n_seq ? offsets[i + 1] : 0;
    start = min(max(a, 0), T);
    len = max(min(max(b, 0), T) - start, 0);
    return (len + BQ - 1) / BQ;
  };
  Work w{0, 0, 0};
  int start, len, nt, pick = -1, tile = 0;
  if (n_seq <= 64) {
    nt = lane_seq(0, start, len);
    int lo = 0, hi = (T + BQ - 1) / BQ, more = 0;  // F(lo) > id >= F(hi) = more
    if (wave_sum_i(nt) <= id) return w;
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
    int before = 0;
    for (int first = 0; first < n_seq; first += 64) {
      nt = lane_seq(first, start, len);
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

template <int DH, int NQ>
__global__ __launch_bounds__(256, NQ == 2 ? 1 : DH == 64 ? 3 : 2) void attention_packed_kernel(PackedAttn a) {
  constexpr int ROWB = DH * 2, TILE = BKV * ROWB, LOADS = TILE / 1024 / 4;  // 1 KB loads a wave and tile of K or V
  constexpr int RPK = 1024 / ROWB, CPR = ROWB / 16;                         // rows a load, 16-byte chunks a row
  constexpr int ND = DH / 32, KS = DH / 16, BQ = 128 * NQ;
  // one array per operand and stage: the compiler can tell reads from the loads into other arrays
  __shared__ __attribute__((aligned(1024))) char sk0[TILE];
  __shared__ __attribute__((aligned(1024))) char sk1[TILE];
  __shared__ __attribute__((aligned(1024))) char sv0[TILE];
  __shared__ __attribute__((aligned(1024))) char sv1[TILE];

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = lane >> 5, li = lane & 31;
  const int ti = div_by(blockIdx.x, a.by_H), hr = blockIdx.x - ti * a.H;
  // heads of a KV head H / Hkv ids apart ... 8 ids side by side go to 8 XCDs
  const int gi = div_by(hr, a.by_Hkv), hk = hr - gi * a.Hkv, h = hk * a.G + gi;
  const Work wk = work_of(a.offsets, a.n_seq, a.T, ti, BQ);
  if (wk.len == 0) return;
  const int L = wk.len, q0 = wk.q0, qw0 = q0 + wave * 32 * NQ;

  const bf16_t* kh = (const bf16_t*)a.k.p + (int64_t)wk.start * a.k.token + hk * a.k.head;
  const bf16_t* vh = (const bf16_t*)a.v.p + (int64_t)wk.start * a.v.token + hk * a.v.head;

  // the wave's queries as MFMA B operands; lanes past L load row L - 1 (not stored)
  bf16x8 fq[NQ][KS];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const bf16_t* row = (const bf16_t*)a.q.p + (int64_t)(wk.start + min(qw0 + n * 32 + li, L - 1)) * a.q.token + h * a.q.head;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) fq[n][ks] = *(const bf16x8*)(row + ks * 16 + half * 8);
  }
  const int ntiles = (min(L, q0 + BQ) + BKV - 1) / BKV;
  const int mine = min(qw0, L - 1) / BKV;  // the wave's last tile; waves without queries follow the last one that has
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
    for (int j = 0; j < LOADS; ++j) dma16(r, st + (wave * LOADS + j) * 1024, kv[j], 0);
  };
  auto issue_v = [&](char* st, int t) {
    const __amdgpu_buffer_rsrc_t r = rows_at(vh, a.v.token, t);
#pragma unroll
    for (int j = 0; j < LOADS; ++j) dma16(r, st + (wave * LOADS + j) * 1024, vv, (int)(j * RPK * a.v.token * 2));
  };

  f32x16 acc[NQ][ND];
#pragma unroll
  for (int n = 0; n < NQ; ++n)
#pragma unroll
    for (int t = 0; t < ND; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[n][t][r] = 0.f;
  float m[NQ], l[NQ];
#pragma unroll
  for (int n = 0; n < NQ; ++n) m[n] = -INFINITY, l[n] = 0.f;

  // K tile t + 2 and V tile t + 1 go out at the head of tile t, into the stages that tile t - 1 read last
  issue_k(sk0, 0);
  issue_k(sk1, 1);
  issue_v(sv0, 0);

  f32x16 sa[NQ][2], sb[NQ][2];  // scores of the tile in work and of the next
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
        const bf16x8 f = kfrag(sk0, t, ks);
#pragma unroll
        for (int n = 0; n < NQ; ++n)
          sa[n][t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, fq[n][ks], ks == 0 ? zero : sa[n][t], 0, 0, 0);
      }
  }
  const bf16x2 ones = {(__bf16)1.f, (__bf16)1.f}, none = {(__bf16)0.f, (__bf16)0.f};

  // the maximum of a set's scores; moves the running one where a score is 8 (in log2) above it
  auto raise = [&](int n, const f32x16(&s)[2]) {
    float top = fmaxf(s[0][0], s[1][0]);
#pragma unroll
    for (int r = 1; r < 16; ++r) top = fmaxf(fmaxf(top, s[0][r]), s[1][r]);
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
    top = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])) * a.scale_log2;
    if (__any(top > m[n] + 8.f)) {
      // by the query's own scores alone: its bits do not depend on its neighbours
      const float mn = top > m[n] + 8.f ? top : m[n], f = m[n] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[n] - mn);
      l[n] *= f;
#pragma unroll
      for (int t = 0; t < ND; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[n][t][r] *= f;
      m[n] = mn;
    }
  };
  // weights x, x + 1 of a set (x = 16 t + r) as a bf16 pair, added to its sum
  auto weigh = [&](int n, const f32x16(&s)[2], int x) {
    const float p0 = __builtin_amdgcn_exp2f(fmaf(s[x >> 4][x & 15], a.scale_log2, -m[n]));
    const float p1 = __builtin_amdgcn_exp2f(fmaf(s[x >> 4][(x & 15) + 1], a.scale_log2, -m[n]));
    const bf16x2 w = {(__bf16)p0, (__bf16)p1};
    l[n] = __builtin_amdgcn_fdot2_f32_bf16(w, ones, l[n], false);
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
  auto body = [&](auto S_, int it, f32x16(&s)[NQ][2], f32x16(&sn)[NQ][2]) {
    constexpr int S = decltype(S_)::value;
    // K tile it + 1 and V tile it landed, and every wave is done with the stages that the next loads overwrite
    landed();
    char* vst = S == 0 ? sv0 : sv1;
    const char* kst = S == 0 ? sk1 : sk0;
    if (it + 1 < ntiles) {
      issue_k(S == 0 ? sk0 : sk1, it + 2);
      issue_v(S == 0 ? sv1 : sv0, it + 1);
    }
    if (work && it < mine) {
      uint32_t p[NQ][16];
      // operands in order: the next tile's K (NK), then this tile's V; read LA ahead of the MFMAs that take them.
      // The scheduling barriers let only VALU and scalar instructions cross, so this order is the one issued.
      constexpr int NK = 2 * KS, NV = 4 * ND, LA = 4, PPK = 16 / NK > 0 ? 16 / NK : 1;
      bf16x8 fr[LA];
      auto fetch = [&](int i) {
        if (i < NK)
          fr[i % LA] = kfrag(kst, i & 1, i >> 1);
        else if (i < NK + NV)
          fr[i % LA] = vfrag(vst, (i - NK) / ND, (i - NK) % ND);
      };
#pragma unroll
      for (int i = 0; i < LA; ++i) fetch(i);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int n = 0; n < NQ; ++n) raise(n, s[n]);
#pragma unroll
      for (int i = 0; i < NK; ++i) {
        const int ks = i >> 1, t = i & 1;
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
          sn[n][t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr[i % LA], fq[n][ks], ks == 0 ? zero : sn[n][t], 0, 0, 0);
          if (n == NQ - 1) fetch(i + LA);
#pragma unroll
          for (int x = i * PPK; x < (i + 1) * PPK; ++x) p[n][x] = weigh(n, s[n], 2 * x);
          __builtin_amdgcn_sched_barrier(0x406);
        }
      }
#pragma unroll
      for (int c4 = 0; c4 < 4; ++c4)
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) {
          const int i = NK + c4 * ND + dt;
#pragma unroll
          for (int n = 0; n < NQ; ++n) {
            acc[n][dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr[i % LA], operand(p[n] + 4 * c4), acc[n][dt], 0, 0, 0);
            if (n == NQ - 1) fetch(i + LA);
            __builtin_amdgcn_sched_barrier(0x406);
          }
        }
    }
  };
  for (int base = 0; base < ntiles; base += 2) {
    body(std::integral_constant<int, 0>{}, base, sa, sb);
    if (base + 1 < ntiles) body(std::integral_constant<int, 1>{}, base + 1, sb, sa);
  }
  if (!work) return;
  // the last two tiles' values are both still there
  char* const vst = mine & 1 ? sv1 : sv0;
  if (mine & 1)
#pragma unroll
    for (int n = 0; n < NQ; ++n) sa[n][0] = sb[n][0], sa[n][1] = sb[n][1];
  // the wave's last tile: of a set, the keys of half `diag` up to its own, those of the half before it, none after
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const int diag = NQ == 2 ? n : wave & 1;
    uint32_t p[16];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int key = t * 32 + (r >> 2) * 8 + half * 4 + (r & 3);
        sa[n][t][r] = key <= diag * 32 + li ? sa[n][t][r] : -INFINITY;
      }
    raise(n, sa[n]);
#pragma unroll
    for (int x = 0; x < 16; ++x) p[x] = weigh(n, sa[n], 2 * x);
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
        if (dirty) mark(acc[n], vst, t);
      }
#pragma unroll
      for (int i = 0; i < 2 * ND; ++i) {
        bf16x8 f = vfrag(vst, 2 * t + i / ND, i % ND);
        if (dirty) f = without(f, nullptr);
        acc[n][i % ND] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, operand(p + 4 * (2 * t + i / ND)), acc[n][i % ND], 0, 0, 0);
        if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);
      }
    }
  }

#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const float total = l[n] + __shfl_xor(l[n], 32, 64);
    const int qi = qw0 + n * 32 + li;
    if (qi < L) {
      const float inv = 1.f / total;
      bf16_t* row = (bf16_t*)a.o.p + (int64_t)(wk.start + qi) * a.o.token + h * a.o.head;
#pragma unroll
      for (int dt = 0; dt < ND; ++dt)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          *(u32x2*)(row + dt * 32 + g * 8 + half * 4) =
              u32x2{pack_bf2(acc[n][dt][g * 4 + 0] * inv, acc[n][dt][g * 4 + 1] * inv),
                    pack_bf2(acc[n][dt][g * 4 + 2] * inv, acc[n][dt][g * 4 + 3] * inv)};
    }
  }
}

template <int DH, int NQ>
hipError_t launch(const PackedAttn& a, hipStream_t s) {
  // every tile but a prompt's last has 128 NQ queries
  const int64_t tiles = (int64_t)a.T / (128 * NQ) + a.n_seq, wgs = tiles * a.H;
  if (wgs >= 1ll << 24) return hipErrorInvalidValue;  // fewer than 2^32 threads
  hipLaunchKernelGGL((attention_packed_kernel<DH, NQ>), dim3((unsigned)wgs), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t attention_packed(PackedAttn a, int dh, hipStream_t s) {
  a.G = a.H / a.Hkv;
  a.by_H = fast_div(a.H);
  a.by_Hkv = fast_div(a.Hkv);
  a.scale_log2 = 1.4426950408889634f / sqrtf((float)dh);
  return dh == 128 ? launch<128, 1>(a, s) : launch<64, 1>(a, s);
}

}  // namespace vla
