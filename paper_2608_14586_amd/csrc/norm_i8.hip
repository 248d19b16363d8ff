// Rows into 8-bit codes with a scale each, behind the residual's addition and
// the RMS norm where they are asked for:
//   t = x + add,  u = t g,  a = max |u|,  code = 127 u / a to the nearest, ties to even,
//   scale = a / 127 / sqrt(mean(t^2) + eps)     (without a gain u = t, scale = a / 127)
// The norm's factor is the same along a row, so the codes do without it and with
// the scale alone it comes in: one pass over the row, both reductions at once.
//
// t and u are fp32 numbers, and a code is the one that the quotient of these
// numbers as they are rounds to.  In fp32 it is within 2^-15 of that quotient (q =
// u (127 / a), two roundings, |q| <= 127), so one that lies no nearer to a border
// k + 1/2 is right; for the others, one in 10^4, 254 u - (2 k + 1) a decides, whose
// terms are exact in 64 bits.
//
// Bound by memory: the row stays in registers between its reductions and its
// codes.  2048 rows of 4096, the fp32 residual with a bf16 addition, written back, 92 MB:
// 19.8 us (4.7 TB/s, the launch's 2.3 us included), 23 with nothing in a cache; 1777 rows
// of 11008 in bf16 without a gain 14.0; 4 rows 2.9, which is the launch.
//
// The sum of squares is fp32.  Where it leaves what fp32 holds well (rows near 2^64 and
// above, or 2^-40 and below) it is taken again in 64 bits.
#include "kernels.h"

namespace vla {
namespace {

__device__ __forceinline__ void load8(const void* p, int64_t at, bool f32, float (&x)[8]) {
  if (f32) {
    const f32x4 a = *(const f32x4*)((const float*)p + at), b = *(const f32x4*)((const float*)p + at + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = a[e], x[4 + e] = b[e];
  } else {
    const u32x4 w = *(const u32x4*)((const bf16_t*)p + at);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[2 * e] = __uint_as_float(w[e] << 16);
      x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
    }
  }
}

constexpr float BORDER = 0.5f - 0x1p-15f;

__device__ __forceinline__ uint32_t pack4(const float* c) {
  const uint32_t lo = ((uint32_t)(int)c[0] & 255u) | ((uint32_t)(int)c[1] & 255u) << 8;
  const uint32_t hi = ((uint32_t)(int)c[2] & 255u) | ((uint32_t)(int)c[3] & 255u) << 8;
  return lo | hi << 16;
}

__device__ __forceinline__ double wave_sum(double x) {
#pragma unroll
  for (int m = 32; m; m >>= 1) x += __shfl_xor(x, m, 64);
  return x;
}

// One row per workgroup of T threads, NV pieces of 8 values a thread; NORM: with a gain.
template <int T, int NV, bool NORM>
__global__ __launch_bounds__(T) void norm_i8_kernel(NormI8Args p) {
  constexpr int W = T / 64;
  __shared__ uint32_t tops[W];
  __shared__ float sums[W];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t row = blockIdx.x;
  const int nv = p.d >> 3;
  float u[NV][8];
  float ss = 0.f;
  uint32_t top = 0;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int i = tid + v * T;
    if (i < nv) {
      load8(p.x, row * p.ldx + i * 8, p.x_f32, u[v]);
      if (p.add) {
        float y[8];
        load8(p.add, row * p.ldadd + i * 8, p.add_f32, y);
#pragma unroll
        for (int e = 0; e < 8; ++e) u[v][e] += y[e];
      }
    }
  }
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int i = tid + v * T;
    if (i < nv) {
      if (p.sum) {
        float* s = p.sum + row * p.ldsum + i * 8;
        *(f32x4*)s = f32x4{u[v][0], u[v][1], u[v][2], u[v][3]};
        *(f32x4*)(s + 4) = f32x4{u[v][4], u[v][5], u[v][6], u[v][7]};
      }
      if constexpr (NORM) {
        float g[8];
        load8(p.g, i * 8, true, g);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          ss = fmaf(u[v][e], u[v][e], ss);
          u[v][e] *= g[e];
        }
      }
      // magnitudes as whole numbers: infinities are above all finite ones, NaN above those
#pragma unroll
      for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(u[v][e]) & 0x7fffffffu);
    }
  }
  top = wave_max_u(top);
  if constexpr (NORM) ss = warp_sum(ss);
  if constexpr (W > 1) {
    if (lane == 0) {
      tops[wave] = top;
      if constexpr (NORM) sums[wave] = ss;
    }
    __syncthreads();
    top = tops[0];
    if constexpr (NORM) ss = sums[0];
#pragma unroll
    for (int w = 1; w < W; ++w) {
      top = max(top, tops[w]);
      if constexpr (NORM) ss += sums[w];
    }
  }
  const bool finite = top < 0x7f800000u;
  float a = __uint_as_float(top);
  if (!finite || a < 0x1p-100f) a = 0.f;  // codes of zero, the scale NaN or zero
  const float inv = a > 0.f ? 127.f / a : 0.f;
  const bool again = NORM && a > 0.f && !(ss >= 0x1p-80f && ss < INFINITY);
  double sq = 0.0;
  if (again) {  // the whole workgroup
    __shared__ double wide[W];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int i = tid + v * T;
      if (i >= nv) continue;
      float t[8], y[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      if (p.sum) {  // what this thread wrote; x or add may be the same memory
        load8(p.sum, row * p.ldsum + i * 8, true, t);
      } else {
        load8(p.x, row * p.ldx + i * 8, p.x_f32, t);
        if (p.add) load8(p.add, row * p.ldadd + i * 8, p.add_f32, y);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) sq += (double)(t[e] + y[e]) * (double)(t[e] + y[e]);
    }
    sq = wave_sum(sq);
    if (lane == 0) wide[wave] = sq;
    __syncthreads();
    sq = 0.0;
#pragma unroll
    for (int w = 0; w < W; ++w) sq += wide[w];
  }
  if (tid == 0) {
    float s = a * (1.f / 127.f);
    if (NORM && a > 0.f) {
      if (again)  // the factor alone may leave fp32, the scale does not for it
        s = (float)(s / sqrt(sq / p.d + (double)p.eps));
      else
        s *= 1.f / sqrtf(ss / (float)p.d + p.eps);
    }
    p.scales[row] = finite ? s : __uint_as_float(0x7fc00000u);
  }
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int i = tid + v * T;
    if (i >= nv) continue;
    float c[8], far = 0.f;
    if (a == 0.f) {  // NaN times zero is none
#pragma unroll
      for (int e = 0; e < 8; ++e) c[e] = 0.f;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float q = u[v][e] * inv;
        c[e] = rintf(q);
        far = fmaxf(far, fabsf(q - c[e]));
      }
      if (far > BORDER) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float q = u[v][e] * inv, k = floorf(q);
          if (fabsf(q - c[e]) > BORDER) {
            const double side = 254.0 * (double)u[v][e] - (2.0 * (double)k + 1.0) * (double)a;
            c[e] = side > 0.0 || (side == 0.0 && ((int)k & 1)) ? k + 1.f : k;
          }
        }
      }
    }
    *(u32x2*)(p.codes + row * p.ldc + i * 8) = u32x2{pack4(c), pack4(c + 4)};
  }
}

template <int T, int NV>
hipError_t launch(const NormI8Args& a, int M, hipStream_t s) {
  if (a.g)
    hipLaunchKernelGGL((norm_i8_kernel<T, NV, true>), dim3(M), dim3(T), 0, s, a);
  else
    hipLaunchKernelGGL((norm_i8_kernel<T, NV, false>), dim3(M), dim3(T), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t norm_i8(const NormI8Args& a, int M, hipStream_t s) {
  const int nv = a.d / 8;
  if (nv <= 64) return launch<64, 1>(a, M, s);
  if (nv <= 128) return launch<128, 1>(a, M, s);
  if (nv <= 256) return launch<256, 1>(a, M, s);
  if (nv <= 512) return launch<256, 2>(a, M, s);
  if (nv <= 1024) return launch<512, 2>(a, M, s);
  if (nv <= 1536) return launch<512, 3>(a, M, s);
  if (nv <= 2048) return launch<512, 4>(a, M, s);
  return nv <= 4096 ? launch<1024, 4>(a, M, s) : hipErrorInvalidValue;
}

}  // namespace vla
