/*
 * vla_ops.h -- operator-level entry points of the VLA prefix library.
 *
 * The kernels that vla_prefix.h's block calls are built from, exposed one by
 * one on caller-owned DEVICE pointers so each can be checked and timed alone.
 * All are enqueued on `stream` (a hipStream_t as void*, NULL = the null
 * stream) and return after launch; shapes are validated first and a rejected
 * call launches nothing (VLA_ERR_INVALID_ARG / VLA_ERR_UNSUPPORTED).
 * bf16 = bfloat16 bit patterns.  Row-major, innermost index last.
 */
#ifndef VLA_OPS_H
#define VLA_OPS_H

#include "vla_prefix.h"

#ifdef __cplusplus
extern "C" {
#endif

/* C[M][N] (fp32) = A[M][K] (bf16) * W[N][K]^T (bf16): the projection of every
 * block's linear layers (bf16 MFMA, fp32 accumulation).  K % 64 == 0. */
vla_status vla_op_gemm_bf16(const void *A, const void *W, float *C, int M, int N, int K, void *stream);

/* Scaled dot-product attention of the blocks: o[B][L][H*dh] (bf16) =
 * softmax(q k^T / sqrt(dh), causal mask if `causal`) v per (b, head), query
 * head h reading KV head h / (H / Hkv).  q[B][H][L][dh], k[B][Hkv][L][dh],
 * vt[B][Hkv][dh][ldvt] = V transposed with the keys of every group of 16
 * stored in the order [0-3, 8-11, 4-7, 12-15] (column c holds key c with
 * bits 2 and 3 swapped), the order the MFMA consumes them; ldvt >= L rounded
 * up to 16, ldvt % 16 == 0; columns of keys >= L are never used.  All bf16.  dh in {64, 128}. */
vla_status vla_op_attention_bf16(const void *q, const void *k, const void *vt, int ldvt, void *o, int B, int H,
                                 int Hkv, int L, int dh, int causal, void *stream);

/* The fused-epilogue products below take their weights packed slab-major,
 * the layout the resident block weights use: W[N][K] (bf16 rows) cut into
 * slabs of 128 rows x 64 k, each one contiguous block,
 *   element (n, k) at ((k / 64 * nblk + n / 128) * 128 + n % 128) * 64 + k % 64,
 * nblk = N rounded up to a multiple of 256, divided by 128 (pad rows zero).
 * vla_op_packed_weight_elems gives the element count (0 for a shape the
 * products reject: N <= 0, K <= 0, K % 64 != 0);
 * vla_op_pack_weight_bf16 packs HOST row-major W into HOST memory Wp of
 * that many elements (no GPU work). */
size_t vla_op_packed_weight_elems(int N, int K);
vla_status vla_op_pack_weight_bf16(const void *W, void *Wp, int N, int K);

/* H[M][N] (fp32, in place) += A[M][K] (bf16) * W^T + bias[N] (fp32, NULL =
 * none), Wp packed as above: the residual products of the blocks (output
 * projection, down / fc2).  Each lane reads the residual of its accumulators
 * behind the last K slab; bias and residual are added in the accumulators
 * and the sums stored from them.  N % 4 == 0, K % 64 == 0. */
vla_status vla_op_gemm_residual_bf16(const void *A, const void *Wp, float *H, const float *bias, int M, int N, int K,
                                     void *stream);

/* out[M][N] (bf16) = f(A[M][K] * W^T + bias[N]), Wp packed as above, bias
 * fp32 or NULL, f = the exact GELU z * Phi(z) (erfc by Abramowitz & Stegun
 * 7.1.26, |error| <= 1.5e-7) when `gelu`, else the identity: the ViT fc1
 * product and the plain bias product.  N % 8 == 0, K % 64 == 0. */
vla_status vla_op_gemm_bias_bf16(const void *A, const void *Wp, void *out, const float *bias, int M, int N, int K,
                                 int gelu, void *stream);

/* How a product of the blocks runs, for tests and timings.  vla_op_gemm_route
 * (host only, no GPU work): columns [0, *n1) in tiles of first[0] rows x
 * first[1] columns by first[2] waves, the rest, if *n1 < N, in a second launch
 * in tiles `second` (zeros if there is none); a_parts = 2 for a split operand.
 * vla_op_gemm_tile_bf16 runs VLA_GEMM_RESIDUAL, _BIAS or _GELU (the
 * arguments of the two entry points above) in the tile of these sizes
 * whatever the choice; VLA_ERR_UNSUPPORTED if the product has no such tile,
 * or only for whole multiples of its columns. */
typedef enum {
  VLA_GEMM_F32 = 0,      /* vla_op_gemm_bf16 */
  VLA_GEMM_RESIDUAL = 1, /* output projection, down, fc2, patch embedding */
  VLA_GEMM_BIAS = 2,     /* connector, second product */
  VLA_GEMM_GELU = 3,     /* fc1; connector, first product */
  VLA_GEMM_SWIGLU = 4,   /* gate/up (N = 2 d_ff, padded) */
  VLA_GEMM_QKV = 5
} vla_gemm_op;
vla_status vla_op_gemm_route(int op, int M, int N, int K, int a_parts, int first[3], int *n1, int second[3]);
vla_status vla_op_gemm_tile_bf16(int op, int rows, int cols, int waves, const void *A, const void *Wp, void *out,
                                 const float *bias, int M, int N, int K, void *stream);

/* y[M][d] (bf16) = RMSNorm(x[M][d] fp32; gain g[d] fp32, eps) -- or
 * LayerNorm with shift b[d] when b != NULL.  d % 4 == 0, d <= 8192. */
vla_status vla_op_norm_bf16(const float *x, const float *g, const float *b, float eps, void *y, int M, int d,
                            void *stream);

/* ------------------------------------------------------------------------
 * Decode with 4-bit weights and a 4-bit KV cache.  A block's attention half
 * for new tokens is: vla_op_norm_bf16, vla_op_gemv_w4 (QKV),
 * vla_op_qk_norm_rope, vla_op_kv4_store, vla_op_attention_kv4,
 * vla_op_gemv_w4 (output projection into the residual); its MLP half:
 * vla_op_norm_bf16, vla_op_gemv_w4 with swiglu, vla_op_gemv_w4.  Nothing is
 * allocated, no call keeps state between calls, and all can be captured into
 * a graph.  All pointers belong to the current device.  An argument that is
 * missing, negative or not one of its choices is VLA_ERR_INVALID_ARG; a size,
 * stride or alignment that the kernels do not take VLA_ERR_UNSUPPORTED.  Sizes
 * of zero (rows, sequences, tokens) are valid and launch nothing.  What a call
 * writes overlaps nothing else of it, but where its text allows it.
 */

/* Head rows of several sequences: element (b, t, h, d) lies at
 * p[b * seq + t * token + h * head + d].  Strides are in elements, >= 0 and
 * multiples of 8; p is 16-byte aligned.  So rows inside a fused projection's
 * output, [B][L][heads][dh] and [B][heads][L][dh] are all described in place. */
typedef struct {
  void *p;
  int64_t seq, token, head;
} vla_heads;

/* 4-bit weights: W[n][k] = scales[n][k / group] * (codes[n][k] - zeros[n][k / group]).
 * vla_op_w4_pack lays codes[N][K] (one a byte, the low four bits), scales and
 * zeros [N][ceil(K / group)] (bf16; zeros NULL: 8 everywhere) out for
 * vla_op_gemv_w4, in Wp of vla_op_w4_packed_bytes bytes (16-byte aligned).
 * All DEVICE pointers.  group in {32, 64, 128}, K % 8 == 0 (the last group
 * may be short).  vla_op_w4_packed_bytes is 0 for sizes that are refused. */
size_t vla_op_w4_packed_bytes(int N, int K, int group);
vla_status vla_op_w4_pack(const void *codes, const void *scales, const void *zeros, void *Wp, int N, int K, int group,
                          void *stream);

/* out[M][N] = x[M][K] (bf16) * W^T + residual[M][N] (fp32, NULL = none), W the
 * packed 4-bit weights, out in out_dtype, accumulated in fp32; made for the
 * few rows of a decode step (the weights are read once per 16 rows).
 * swiglu: W holds N / 2 gate rows, then the N / 2 up rows, and out[M][N / 2] =
 * silu(x Wgate^T) * (x Wup^T) + residual; N % 32 == 0.
 * Row strides in elements, no less than a row's width where M > 1: ldx of x (a
 * multiple of 8; x 16-byte aligned), ldo of out and of residual, which may be
 * the same memory (fp32 out).  A row of x that is not finite gives a row of
 * out that is not finite, and reaches no other row. */
vla_status vla_op_gemv_w4(const void *x, int64_t ldx, const void *Wp, const float *residual, void *out, int64_t ldo,
                          vla_dtype out_dtype, int swiglu, int M, int N, int K, int group, void *stream);

/* RMS norm of every query and key head, then the rotary embedding, in one pass
 * over q[B][L][H][dh] and k[B][L][Hkv][dh] (both in_dtype) into q_out, k_out
 * (bf16, same shapes):  y = x * rsqrt(mean(x^2) + eps) * g over the head's dh
 * values, then pairs (y[i], y[i + dh/2]) turned by the angle of the token's
 * position, whose cosines and sines are row pos of cos, sin [n_pos][dh/2].
 * gq[dh], gk[dh] fp32 gains, each NULL = no norm; cos, sin both NULL = no
 * rotation.  pos[B][L] (device int32), NULL = the token's index t; with
 * rotation, a token whose position is not in [0, n_pos) is padding: its rows
 * of q_out and k_out stay as they were.  Gains and tables 16-byte aligned,
 * eps >= 0.
 * q_out and k_out may be q and k themselves (bf16, same strides).  dh in {64, 128}. */
vla_status vla_op_qk_norm_rope(const vla_heads *q, const vla_heads *k, vla_dtype in_dtype, const float *gq,
                               const float *gk, float eps, const float *cos, const float *sin, int n_pos,
                               const int32_t *pos, const vla_heads *q_out, const vla_heads *k_out, int B, int L, int H,
                               int Hkv, int dh, void *stream);

/* A KV cache of 4 bits a value for B sequences of up to L_cap tokens:
 * vla_op_kv4_bytes bytes of device memory (16-byte aligned), sequence by
 * sequence, head by head, opaque within.  Every 32 dims of a key or value row
 * share m = min and s = (max - min) * (1 / 15), an fp32 product rounded to
 * bf16; a value x is held as c = (x - m) / s, the difference rounded to fp32,
 * the quotient to the nearest whole number (ties to even), at most 15, and
 * stands for m + s c.  Groups whose range is below 2^-99 are held as m; groups
 * with a value that is not finite read back as NaN.
 * store puts rows k, v[B][L][Hkv][dh] (bf16) at positions start[b] + t, t <
 * count[b] (device int32; NULL: start 0, count L; count is cut to [0, L]);
 * load takes them out into k, v.  Positions outside [0, L_cap) are left out,
 * and everything else of the cache (store) or of k, v (load) stays as it was.
 * A call may touch one sequence's slot once; calls on one cache must be ordered
 * (one stream).  L_cap % 32 == 0, L_cap <= 2^24, dh in {64, 128}.
 * vla_op_kv4_bytes is 0 for sizes that are refused. */
size_t vla_op_kv4_bytes(int B, int Hkv, int L_cap, int dh);
vla_status vla_op_kv4_store(const vla_heads *k, const vla_heads *v, const int32_t *start, const int32_t *count,
                            void *cache, int B, int L, int Hkv, int L_cap, int dh, void *stream);
vla_status vla_op_kv4_load(const void *cache, const int32_t *start, const int32_t *count, const vla_heads *k,
                           const vla_heads *v, int B, int L, int Hkv, int L_cap, int dh, void *stream);

/* Attention over the 4-bit cache: queries q[B][Lq][H][dh] (bf16) are the last
 * Lq of the lens[b] tokens (device int32) that sequence b's cache holds, their
 * own keys and values stored already; query i stands at position p = lens[b] -
 * Lq + i and o[b][i][h] (bf16) = softmax(q k_j / sqrt(dh)) v_j over the keys
 * j <= p of KV head h / (H / Hkv) -- with window > 0 over those with j > p -
 * window or j < sinks (a sliding window, and first tokens that stay visible).
 * Made for a decode step's few tokens: every 16 queries of a KV head or less
 * read the cache once more.
 * A query that sees no key (p < 0) gives zeros.  Cached rows that no query
 * sees may hold anything.  max_len: no sequence is longer (lens above it, or
 * below 0, are cut), max_len <= L_cap; it decides how the work is split, so
 * the closer the better.  scratch: vla_op_attention_kv4_scratch bytes (may be
 * 0) of device memory, 16-byte aligned, for this call alone until it is done
 * (calls that may run at the same time need one each).  That size never falls
 * with max_len, all else alike: scratch for the longest call serves every
 * shorter one.  VLA_ERR_SHAPE if scratch_bytes is less.  dh in {64, 128}, H %
 * Hkv == 0. */
size_t vla_op_attention_kv4_scratch(int B, int Lq, int H, int Hkv, int dh, int max_len, int window, int sinks);
vla_status vla_op_attention_kv4(const vla_heads *q, const void *cache, const int32_t *lens, const vla_heads *o, int B,
                                int Lq, int H, int Hkv, int L_cap, int dh, int max_len, int window, int sinks,
                                void *scratch, size_t scratch_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* VLA_OPS_H */
