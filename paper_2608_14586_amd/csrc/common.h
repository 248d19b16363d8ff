// Shared device helpers for the gfx950 kernels of the VLA prefix.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

typedef uint16_t bf16_t;  // bfloat16 bit pattern
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

#define VLA_WAVE 64

__device__ __forceinline__ float bf2f(bf16_t b) { return __uint_as_float(((uint32_t)b) << 16); }

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

// float -> bfloat16, round to nearest even (v_cvt_pk_bf16_f32 on gfx950).
__device__ __forceinline__ bf16_t f2bf(float f) { return __builtin_bit_cast(bf16_t, (__bf16)f); }

// two floats -> packed bf16 pair (lo in bits 0..15), one v_cvt_pk_bf16_f32.
__device__ __forceinline__ uint32_t pack_bf2(float lo, float hi) {
  bf16x2_t v = {(__bf16)lo, (__bf16)hi};
  return __builtin_bit_cast(uint32_t, v);
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
  return v;
}

// A value of another lane by DPP: CTRL 0xB1 and 0x4E exchange lanes 1 and 2
// apart, 0x141 and 0x140 mirror a row's halves and the row (16 lanes), so that
// after the first n of the four every 2^n lanes have met.
template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), CTRL, 0xf, 0xf, true));
}
// over the N (4, 8 or 16) lanes that lie side by side
template <int N = 16>
__device__ __forceinline__ float row_max(float x) {
  x = fmaxf(x, dpp<0xB1>(x));
  x = fmaxf(x, dpp<0x4E>(x));
  if constexpr (N > 4) x = fmaxf(x, dpp<0x141>(x));
  if constexpr (N > 8) x = fmaxf(x, dpp<0x140>(x));
  return x;
}
template <int N = 16>
__device__ __forceinline__ float row_sum(float x) {
  x += dpp<0xB1>(x);
  x += dpp<0x4E>(x);
  if constexpr (N > 4) x += dpp<0x141>(x);
  if constexpr (N > 8) x += dpp<0x140>(x);
  return x;
}

// ---- 4-bit codes as MFMA operands (w4.hip, kv4.hip)
__host__ __device__ constexpr uint32_t rotl(uint32_t w, int n) { return w << n | w >> (32 - n); }

// 8 codes of a word as bf16 numbers 16 + c: rotated left by 3, a word's nibbles i
// and 4 + i lie at the top mantissa bits (3-6) of a pair of 16.0, 4 i bits to the right.
// The constants sit in registers of their own, hidden from the compiler: and-or
// takes no literals, and two instructions in its place cost a third of the
// unpacking.
struct UnpackCodes {
  uint32_t bias = 0x41804180u, mask = 0x00780078u;
  __device__ __forceinline__ UnpackCodes() { asm("" : "+s"(bias), "+v"(mask)); }
  __device__ __forceinline__ bf16x8 operator()(uint32_t w) const {
    const u32x4 v = {(w & mask) | bias, (__builtin_amdgcn_alignbit(w, w, 4) & mask) | bias,
                     (__builtin_amdgcn_alignbit(w, w, 8) & mask) | bias,
                     (__builtin_amdgcn_alignbit(w, w, 12) & mask) | bias};
    return __builtin_bit_cast(bf16x8, v);
  }
};
__device__ __forceinline__ f32x4 mfma(const bf16x8& a, const bf16x8& b, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

static constexpr inline int cdiv(int a, int b) { return (a + b - 1) / b; }
