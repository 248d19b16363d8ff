// Operator-level entry points (include/vla_ops.h).
#include <hip/hip_runtime.h>

#include "../../include/vla_ops.h"
#include "kernels.h"

namespace {
vla_status status_of(hipError_t e) {
  if (e == hipSuccess) return VLA_OK;
  return e == hipErrorInvalidValue ? VLA_ERR_UNSUPPORTED : VLA_ERR_HIP;
}
static_assert((int)vla::GemmOp::F32 == VLA_GEMM_F32 && (int)vla::GemmOp::RESIDUAL == VLA_GEMM_RESIDUAL &&
                  (int)vla::GemmOp::BIAS == VLA_GEMM_BIAS && (int)vla::GemmOp::GELU == VLA_GEMM_GELU &&
                  (int)vla::GemmOp::SWIGLU == VLA_GEMM_SWIGLU && (int)vla::GemmOp::QKV == VLA_GEMM_QKV,
              "vla_gemm_op names GemmOp's values");

// ---- checks of the 4-bit operators' arguments
// a launch has fewer than 2^32 threads along x: 2 x 256 (cache rows), 512 or 256 a unit below
constexpr int64_t MAX_GRID = 0x7fffff;
bool aligned(const void* p, uintptr_t n) { return (uintptr_t)p % n == 0; }
bool readable(const vla_heads& h, int B, int L) {
  return (h.p || B == 0 || L == 0) && h.seq >= 0 && h.token >= 0 && h.head >= 0;
}
// rows that are written must not be one and the same
bool writable(const vla_heads& h, int B, int L, int H) {
  return readable(h, B, L) && (B < 2 || h.seq) && (L < 2 || h.token) && (H < 2 || h.head);
}
bool heads_ok(const vla_heads& h) { return aligned(h.p, 16) && h.seq % 8 == 0 && h.token % 8 == 0 && h.head % 8 == 0; }
vla::Heads heads(const vla_heads& h) { return {h.p, h.seq, h.token, h.head}; }

vla_status w4_check(int N, int K, int group) {
  if (N <= 0 || K <= 0) return VLA_ERR_INVALID_ARG;
  if (K % 8 || (group != 32 && group != 64 && group != 128)) return VLA_ERR_UNSUPPORTED;
  if (N > 1 << 25 || K > 1 << 25) return VLA_ERR_UNSUPPORTED;
  return VLA_OK;
}

vla_status kv4_check(int B, int Hkv, int L_cap, int dh) {
  if (B < 0 || Hkv <= 0 || L_cap <= 0) return VLA_ERR_INVALID_ARG;
  if ((dh != 64 && dh != 128) || L_cap % 32 || L_cap > 1 << 24 || (int64_t)B * Hkv > MAX_GRID)
    return VLA_ERR_UNSUPPORTED;
  return VLA_OK;
}

vla_status kv4_rows(const vla_heads* k, const vla_heads* v, const int32_t* start, const int32_t* count, void* cache,
                    int B, int L, int Hkv, int L_cap, int dh, bool out, vla::Kv4Rows* a) {
  if (!k || !v || L < 0 || B < 0 || (B && !cache)) return VLA_ERR_INVALID_ARG;
  if (!(out ? writable(*k, B, L, Hkv) && writable(*v, B, L, Hkv) : readable(*k, B, L) && readable(*v, B, L)))
    return VLA_ERR_INVALID_ARG;
  const vla_status st = kv4_check(B, Hkv, L_cap, dh);
  if (st != VLA_OK) return st;
  if (!heads_ok(*k) || !heads_ok(*v) || !aligned(cache, 16) || !aligned(start, 4) || !aligned(count, 4) ||
      (int64_t)B * Hkv * ((L + 62ll) / 32) > MAX_GRID)
    return VLA_ERR_UNSUPPORTED;
  *a = vla::Kv4Rows{heads(*k), heads(*v), cache, start, count, B, L, Hkv, L_cap, 0, {}, {}};
  return VLA_OK;
}

// window: one that covers max_len tokens hides none, and is taken out here
vla_status attn_check(int B, int Lq, int H, int Hkv, int dh, int max_len, int* window, int* sinks) {
  if (B < 0 || Lq < 0 || H <= 0 || Hkv <= 0 || max_len < 0 || *window < 0 || *sinks < 0) return VLA_ERR_INVALID_ARG;
  if (H % Hkv || (dh != 64 && dh != 128) || max_len > 1 << 24 || (int64_t)Lq * H > MAX_GRID ||
      (int64_t)B * Lq * H > MAX_GRID || (int64_t)B * Hkv > MAX_GRID ||
      (int64_t)Lq * (H / Hkv) > 16 * 65535)  // tiles of at most 16 queries, along the grid's z
    return VLA_ERR_UNSUPPORTED;
  if (*window >= max_len) *window = 0;
  if (*sinks > max_len) *sinks = max_len;
  if (*window == 0) *sinks = 0;
  return VLA_OK;
}
}  // namespace

extern "C" {

vla_status vla_op_gemm_bf16(const void* A, const void* W, float* C, int M, int N, int K, void* stream) {
  if (!A || !W || !C || M < 0 || N < 0 || K <= 0) return VLA_ERR_INVALID_ARG;
  if (K % 64) return VLA_ERR_UNSUPPORTED;
  return status_of(vla::gemm_bf16_store_f32((const bf16_t*)A, K, (const bf16_t*)W, K, C, N, M, N, K,
                                            (hipStream_t)stream));
}

size_t vla_op_packed_weight_elems(int N, int K) {
  if (N <= 0 || K <= 0 || K % 64) return 0;
  return (size_t)vla::slab_blocks(N) * vla::SLAB_N * K;
}

vla_status vla_op_pack_weight_bf16(const void* W, void* Wp, int N, int K) {
  if (!W || !Wp || N <= 0 || K <= 0) return VLA_ERR_INVALID_ARG;
  if (K % 64) return VLA_ERR_UNSUPPORTED;
  vla::pack_slabs((const uint16_t*)W, (uint16_t*)Wp, N, K);
  return VLA_OK;
}

vla_status vla_op_gemm_residual_bf16(const void* A, const void* Wp, float* H, const float* bias, int M, int N, int K,
                                     void* stream) {
  if (!A || !Wp || !H || M < 0 || N <= 0 || K <= 0) return VLA_ERR_INVALID_ARG;
  if (K % 64 || N % 4) return VLA_ERR_UNSUPPORTED;
  const vla::WOperand w{(const bf16_t*)Wp, 0, vla::slab_blocks(N)};
  return status_of(vla::gemm_bf16_residual((const bf16_t*)A, K, w, H, N, bias, M, N, K, (hipStream_t)stream));
}

vla_status vla_op_gemm_bias_bf16(const void* A, const void* Wp, void* out, const float* bias, int M, int N, int K,
                                 int gelu, void* stream) {
  if (!A || !Wp || !out || M < 0 || N <= 0 || K <= 0) return VLA_ERR_INVALID_ARG;
  if (K % 64 || N % 8) return VLA_ERR_UNSUPPORTED;
  const vla::WOperand w{(const bf16_t*)Wp, 0, vla::slab_blocks(N)};
  hipError_t e = gelu ? vla::gemm_bf16_gelu((const bf16_t*)A, K, w, (bf16_t*)out, N, bias, M, N, K, (hipStream_t)stream)
                      : vla::gemm_bf16_bias((const bf16_t*)A, K, w, (bf16_t*)out, N, bias, M, N, K, (hipStream_t)stream);
  return status_of(e);
}

vla_status vla_op_gemm_route(int op, int M, int N, int K, int a_parts, int* first, int* n1, int* second) {
  if (!first || !n1 || !second || op < VLA_GEMM_F32 || op > VLA_GEMM_QKV) return VLA_ERR_INVALID_ARG;
  vla::GemmTile t[2];
  const hipError_t e = vla::gemm_bf16_route((vla::GemmOp)op, M, N, K, a_parts, &t[0], n1, &t[1]);
  if (e != hipSuccess) return status_of(e);
  int* out[2] = {first, second};
  for (int i = 0; i < 2; ++i) out[i][0] = t[i].rows, out[i][1] = t[i].cols, out[i][2] = t[i].waves;
  return VLA_OK;
}

vla_status vla_op_gemm_tile_bf16(int op, int rows, int cols, int waves, const void* A, const void* Wp, void* out,
                                 const float* bias, int M, int N, int K, void* stream) {
  if (!A || !Wp || !out || M < 0 || N <= 0 || K <= 0) return VLA_ERR_INVALID_ARG;
  if (K % 64 || N % (op == VLA_GEMM_RESIDUAL ? 4 : 8)) return VLA_ERR_UNSUPPORTED;
  const vla::WOperand w{(const bf16_t*)Wp, 0, vla::slab_blocks(N)};
  const vla::GemmTile t{rows, cols, waves};
  const bf16_t* a = (const bf16_t*)A;
  hipStream_t s = (hipStream_t)stream;
  switch (op) {
    case VLA_GEMM_RESIDUAL: return status_of(vla::gemm_bf16_residual(a, K, w, (float*)out, N, bias, M, N, K, s, 1, &t));
    case VLA_GEMM_BIAS: return status_of(vla::gemm_bf16_bias(a, K, w, (bf16_t*)out, N, bias, M, N, K, s, &t));
    case VLA_GEMM_GELU: return status_of(vla::gemm_bf16_gelu(a, K, w, (bf16_t*)out, N, bias, M, N, K, s, &t));
    default: return VLA_ERR_INVALID_ARG;
  }
}

vla_status vla_op_attention_bf16(const void* q, const void* k, const void* vt, int ldvt, void* o, int B, int H,
                                 int Hkv, int L, int dh, int causal, void* stream) {
  if (!q || !k || !vt || !o || B < 0 || H <= 0 || Hkv <= 0 || L < 0) return VLA_ERR_INVALID_ARG;
  if (H % Hkv || (dh != 64 && dh != 128) || ldvt < (L + 15) / 16 * 16 || ldvt % 16) return VLA_ERR_UNSUPPORTED;
  return status_of(vla::attention_bf16((const bf16_t*)q, (const bf16_t*)k, (const bf16_t*)vt, ldvt, (bf16_t*)o, B, H,
                                       Hkv, L, dh, causal != 0, (hipStream_t)stream));
}

vla_status vla_op_norm_bf16(const float* x, const float* g, const float* b, float eps, void* y, int M, int d,
                            void* stream) {
  if (!x || !g || !y || M < 0 || d <= 0) return VLA_ERR_INVALID_ARG;
  if (d % 4 || d > 8192) return VLA_ERR_UNSUPPORTED;
  hipError_t e = b ? vla::layernorm_bf16(x, g, b, eps, (bf16_t*)y, M, d, (hipStream_t)stream)
                   : vla::rmsnorm_bf16(x, g, eps, (bf16_t*)y, M, d, (hipStream_t)stream);
  return status_of(e);
}

// ------------------------------------------------- 4-bit weights and KV cache

size_t vla_op_w4_packed_bytes(int N, int K, int group) {
  return w4_check(N, K, group) == VLA_OK ? vla::w4_packed_bytes(N, K, group) : 0;
}

vla_status vla_op_w4_pack(const void* codes, const void* scales, const void* zeros, void* Wp, int N, int K, int group,
                          void* stream) {
  if (!codes || !scales || !Wp) return VLA_ERR_INVALID_ARG;
  const vla_status st = w4_check(N, K, group);
  if (st != VLA_OK) return st;
  if (!aligned(Wp, 16) || !aligned(scales, 2) || !aligned(zeros, 2)) return VLA_ERR_UNSUPPORTED;
  return status_of(vla::w4_pack((const uint8_t*)codes, (const bf16_t*)scales, (const bf16_t*)zeros, Wp, N, K, group,
                                (hipStream_t)stream));
}

vla_status vla_op_gemv_w4(const void* x, int64_t ldx, const void* Wp, const float* residual, void* out, int64_t ldo,
                          vla_dtype out_dtype, int swiglu, int M, int N, int K, int group, void* stream) {
  if (M < 0 || ldx < 0 || ldo < 0 || (out_dtype != VLA_BF16 && out_dtype != VLA_F32) || (M && (!x || !Wp || !out)))
    return VLA_ERR_INVALID_ARG;
  const vla_status st = w4_check(N, K, group);
  if (st != VLA_OK) return st;
  if (ldx % 8 || !aligned(x, 16) || !aligned(Wp, 16) || !aligned(out, out_dtype == VLA_F32 ? 4 : 2) ||
      !aligned(residual, 4) || (swiglu && N % 32))
    return VLA_ERR_UNSUPPORTED;
  if (M > 1 && (ldx < K || ldo < (swiglu ? N / 2 : N))) return VLA_ERR_INVALID_ARG;
  // 16 rows of x lie within 2^31 bytes
  if (M > 16 * 65535 || (M > 1 && ldx > ((1 << 30) - 1 - K) / 15)) return VLA_ERR_UNSUPPORTED;
  if (M == 0) return VLA_OK;
  return status_of(vla::gemv_w4((const bf16_t*)x, ldx, Wp, residual, out, ldo, out_dtype == VLA_F32, swiglu != 0, M, N,
                                K, group, (hipStream_t)stream));
}

vla_status vla_op_qk_norm_rope(const vla_heads* q, const vla_heads* k, vla_dtype in_dtype, const float* gq,
                               const float* gk, float eps, const float* cos, const float* sin, int n_pos,
                               const int32_t* pos, const vla_heads* q_out, const vla_heads* k_out, int B, int L, int H,
                               int Hkv, int dh, void* stream) {
  if (!q || !k || !q_out || !k_out || !cos != !sin || !(eps >= 0.f) || n_pos < 0 || B < 0 || L < 0 || H <= 0 || Hkv <= 0 ||
      (in_dtype != VLA_BF16 && in_dtype != VLA_F32) || !readable(*q, B, L) || !readable(*k, B, L) ||
      !writable(*q_out, B, L, H) || !writable(*k_out, B, L, Hkv))
    return VLA_ERR_INVALID_ARG;
  if ((dh != 64 && dh != 128) || !heads_ok(*q) || !heads_ok(*k) || !heads_ok(*q_out) || !heads_ok(*k_out) ||
      !aligned(gq, 16) || !aligned(gk, 16) || !aligned(cos, 16) || !aligned(sin, 16) || !aligned(pos, 4) ||
      (int64_t)B * L > MAX_GRID || (int64_t)H + Hkv > MAX_GRID)
    return VLA_ERR_UNSUPPORTED;
  if (B == 0 || L == 0) return VLA_OK;
  const vla::QkNormArgs a{heads(*q), heads(*k), heads(*q_out), heads(*k_out), gq, gk, cos, sin, pos, eps, n_pos,
                          B, L, H, Hkv, {}};
  return status_of(vla::qk_norm_rope(a, in_dtype == VLA_F32, dh, (hipStream_t)stream));
}

size_t vla_op_kv4_bytes(int B, int Hkv, int L_cap, int dh) {
  return kv4_check(B, Hkv, L_cap, dh) == VLA_OK ? vla::kv4_bytes(B, Hkv, L_cap, dh) : 0;
}

vla_status vla_op_kv4_store(const vla_heads* k, const vla_heads* v, const int32_t* start, const int32_t* count,
                            void* cache, int B, int L, int Hkv, int L_cap, int dh, void* stream) {
  vla::Kv4Rows a;
  const vla_status st = kv4_rows(k, v, start, count, cache, B, L, Hkv, L_cap, dh, false, &a);
  if (st != VLA_OK || B == 0 || L == 0) return st;
  return status_of(vla::kv4_store(a, dh, (hipStream_t)stream));
}

vla_status vla_op_kv4_load(const void* cache, const int32_t* start, const int32_t* count, const vla_heads* k,
                           const vla_heads* v, int B, int L, int Hkv, int L_cap, int dh, void* stream) {
  vla::Kv4Rows a;
  const vla_status st = kv4_rows(k, v, start, count, (void*)cache, B, L, Hkv, L_cap, dh, true, &a);
  if (st != VLA_OK || B == 0 || L == 0) return st;
  return status_of(vla::kv4_load(a, dh, (hipStream_t)stream));
}

size_t vla_op_attention_kv4_scratch(int B, int Lq, int H, int Hkv, int dh, int max_len, int window, int sinks) {
  if (attn_check(B, Lq, H, Hkv, dh, max_len, &window, &sinks) != VLA_OK || B == 0 || Lq == 0) return 0;
  return vla::kv4_attention_scratch(B, Lq, H, Hkv, dh, max_len, window, sinks);
}

vla_status vla_op_attention_kv4(const vla_heads* q, const void* cache, const int32_t* lens, const vla_heads* o, int B,
                                int Lq, int H, int Hkv, int L_cap, int dh, int max_len, int window, int sinks,
                                void* scratch, size_t scratch_bytes, void* stream) {
  if (!q || !o || B < 0 || Lq < 0 || !readable(*q, B, Lq) || !writable(*o, B, Lq, H) || (B && (!cache || !lens)))
    return VLA_ERR_INVALID_ARG;
  vla_status st = attn_check(B, Lq, H, Hkv, dh, max_len, &window, &sinks);
  if (st == VLA_OK) st = kv4_check(B, Hkv, L_cap, dh);
  if (st != VLA_OK) return st;
  if (max_len > L_cap) return VLA_ERR_SHAPE;
  if (!heads_ok(*q) || !heads_ok(*o) || !aligned(cache, 16) || !aligned(scratch, 16) || !aligned(lens, 4))
    return VLA_ERR_UNSUPPORTED;
  if (B == 0 || Lq == 0) return VLA_OK;
  if (!scratch && scratch_bytes) return VLA_ERR_INVALID_ARG;
  const vla::Kv4Attn a{heads(*q), heads(*o), cache, lens, (float*)scratch, B, Lq, H, Hkv, L_cap, max_len, window, sinks,
                       0, 0, 0, {}, {}, {}, {}, 0.f};
  const hipError_t e = vla::kv4_attention(a, dh, scratch_bytes, (hipStream_t)stream);
  return e == hipErrorOutOfMemory ? VLA_ERR_SHAPE : status_of(e);
}

}  // extern "C"
