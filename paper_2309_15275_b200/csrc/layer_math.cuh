// The elementwise part of a layer's epilogue: activations, their derivatives, and dropout
// from a counter-based generator.
//
// bf16 data: the activations go through the approximate exponential and reciprocal of the
// special-function unit, with errors far below the rounding of the result (2^-9 of it);
// fp32 data: through CUDA's math functions.  Both take +-infinity to the limit and keep NaN.
#pragma once

#include <cuda_bf16.h>
#include <stdint.h>

#include <type_traits>

#include "lbp_internal.h"
#include "wht_device.cuh"

namespace lbp {
namespace layer {

// ---- numbers --------------------------------------------------------------------------
// What a kernel is handed of an lbp_epilogue's dropout.
struct Drop {
  uint64_t seed, offset;
  const uint64_t *seed_dev, *offset_dev;
  uint64_t* used;
  uint32_t above;   // an element stays where its number, as the high half of a word, is above this
  float scale;
  int32_t on;
};

// ... and what its threads hold.
struct Stream {
  uint32_t k0, k1, c2, c3;
};
__device__ __forceinline__ Stream open_stream(const Drop& d) {
  const uint64_t seed = d.seed_dev != nullptr ? *d.seed_dev : d.seed;
  const uint64_t offset = d.offset + (d.offset_dev != nullptr ? *d.offset_dev : 0ull);
  return Stream{static_cast<uint32_t>(seed), static_cast<uint32_t>(seed >> 32), static_cast<uint32_t>(offset),
                static_cast<uint32_t>(offset >> 32) + 0x80000000u};
}
// (one thread of the grid)
__device__ __forceinline__ void note_used(const Drop& d) {
  if (d.used == nullptr) return;
  const uint64_t seed = d.seed_dev != nullptr ? *d.seed_dev : d.seed;
  const uint64_t offset = d.offset + (d.offset_dev != nullptr ? *d.offset_dev : 0ull);
  d.used[0] = seed;
  d.used[1] = offset;
}

// Philox4x32-10 (Salmon et al. 2011): the numbers of elements 8 group .. 8 group + 7, two a word.
__device__ __forceinline__ uint4 philox(const Stream& s, uint64_t group) {
  uint32_t c0 = static_cast<uint32_t>(group), c1 = static_cast<uint32_t>(group >> 32), c2 = s.c2, c3 = s.c3;
  uint32_t k0 = s.k0, k1 = s.k1;
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t a = static_cast<uint64_t>(c0) * 0xD2511F53u, b = static_cast<uint64_t>(c2) * 0xCD9E8D57u;
    c0 = static_cast<uint32_t>(b >> 32) ^ c1 ^ k0;
    c1 = static_cast<uint32_t>(b);
    c2 = static_cast<uint32_t>(a >> 32) ^ c3 ^ k1;
    c3 = static_cast<uint32_t>(a);
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return make_uint4(c0, c1, c2, c3);
}
// Drops among the elements whose numbers are the low and the high half of w.
__device__ __forceinline__ void drop2(float& lo, float& hi, uint32_t w, const Drop& d) {
  lo = (w << 16) > d.above ? lo * d.scale : 0.f;
  hi = w > d.above ? hi * d.scale : 0.f;
}
// Elements n .. n + 7 (n a multiple of 8), or n .. n + 3 (of 4).
__device__ __forceinline__ void drop(float (&v)[8], uint64_t n, const Stream& s, const Drop& d) {
  const uint4 w = philox(s, n >> 3);
  drop2(v[0], v[1], w.x, d);
  drop2(v[2], v[3], w.y, d);
  drop2(v[4], v[5], w.z, d);
  drop2(v[6], v[7], w.w, d);
}
__device__ __forceinline__ void drop(float (&v)[4], uint64_t n, const Stream& s, const Drop& d) {
  const uint4 w = philox(s, n >> 3);
  const bool upper = (n & 4u) != 0;
  drop2(v[0], v[1], upper ? w.z : w.x, d);
  drop2(v[2], v[3], upper ? w.w : w.y, d);
}

// ---- activations ------------------------------------------------------------------------
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float rcp(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// max and min that keep NaN
__device__ __forceinline__ float at_least(float x, float lo) {
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(x), "f"(lo));
  return y;
}
__device__ __forceinline__ float at_most(float x, float hi) {
  float y;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(x), "f"(hi));
  return y;
}

constexpr float kLog2e = 1.4426950408889634f;
// 2 sqrt(2/pi) and 0.044715 times that: gelu_tanh(z) = z / (1 + exp(-(A z + B z^3)))
constexpr float kTanhA = 1.5957691216057308f, kTanhB = 0.071354816272600247f;

// Phi(-a) = exp(-a^2/2) Q(t) with t = 1 / (1 + 0.38 a): a polynomial of degree 5 fitted to
// exp(a^2/2) erfc(a / sqrt 2) / 2 in the relative error, 3.7e-5 at most over a = 0..40.  Also
// hands out e = exp(-a^2/2).
__device__ __forceinline__ float upper_tail(float a, float* e) {
  const float t = rcp(fmaf(0.38f, a, 1.f));
  *e = ex2(a * (a * (-0.5f * kLog2e)));
  float q = -0.0906074270606041f;
  q = fmaf(q, t, 0.1908050775527954f);
  q = fmaf(q, t, 0.08993600308895111f);
  q = fmaf(q, t, 0.15882457792758942f);
  q = fmaf(q, t, 0.15100638568401337f);
  q = fmaf(q, t, 1.705829163256567e-05f);
  return q * *e;
}

// FAST: for results that are rounded to bf16.
template <int ACT, bool FAST>
__device__ __forceinline__ float act(float z) {
  if constexpr (ACT == LBP_ACT_NONE) {
    return z;
  } else if constexpr (ACT == LBP_ACT_RELU) {
    return at_least(z, 0.f);
  } else if constexpr (ACT == LBP_ACT_GELU) {
    if constexpr (FAST) {
      const float a = at_most(fabsf(z), 100.f);
      float e;
      const float tail = upper_tail(a, &e);
      return fmaf(-a, tail, fmaxf(z, 0.f));   // (a NaN comes through a)
    } else {
      const float c = at_least(z, -100.f);
      return 0.5f * c * erfcf(c * -0.70710678118654752f);
    }
  } else if constexpr (ACT == LBP_ACT_GELU_TANH) {
    const float c = at_least(z, -30.f);
    const float u = c * fmaf(kTanhB, c * c, kTanhA);
    if constexpr (FAST)
      return c * rcp(1.f + ex2(-kLog2e * u));
    else
      return c / (1.f + expf(-u));
  } else {
    const float c = at_least(z, -100.f);
    if constexpr (FAST)
      return c * rcp(1.f + ex2(-kLog2e * c));
    else
      return c / (1.f + expf(-c));
  }
}

template <int ACT, bool FAST>
__device__ __forceinline__ float act_slope(float z) {
  constexpr float kInvSqrt2Pi = 0.3989422804014327f;
  if constexpr (ACT == LBP_ACT_NONE) {
    return 1.f;
  } else if constexpr (ACT == LBP_ACT_RELU) {
    return z > 0.f ? 1.f : z <= 0.f ? 0.f : z;   // (NaN stays)
  } else if constexpr (ACT == LBP_ACT_GELU) {
    if constexpr (FAST) {
      const float c = at_most(at_least(z, -100.f), 100.f);
      float e;
      const float tail = upper_tail(fabsf(c), &e);
      return fmaf(c * kInvSqrt2Pi, e, c > 0.f ? 1.f - tail : tail);
    } else {
      const float c = at_most(at_least(z, -100.f), 100.f);
      return fmaf(c * kInvSqrt2Pi, expf(-0.5f * c * c), 0.5f * erfcf(c * -0.70710678118654752f));
    }
  } else if constexpr (ACT == LBP_ACT_GELU_TANH) {
    // s (1 + z (1 - s) u') with s = 1 / (1 + exp(-u))
    const float c = at_most(at_least(z, -12.f), 12.f);   // (s is 0 and 1 there)
    const float c2 = c * c;
    const float u = c * fmaf(kTanhB, c2, kTanhA), du = fmaf(3.f * kTanhB, c2, kTanhA);
    const float e = FAST ? ex2(-kLog2e * u) : expf(-u);
    const float s = FAST ? rcp(1.f + e) : 1.f / (1.f + e);
    return fmaf(c * du, s * (1.f - s), s);
  } else {
    const float c = at_most(at_least(z, -100.f), 100.f);   // (s is 0 and 1 there)
    const float e = FAST ? ex2(-kLog2e * c) : expf(-c);
    const float s = FAST ? rcp(1.f + e) : 1.f / (1.f + e);
    return fmaf(c, s * (1.f - s), s);
  }
}

// ---- vectors of 16 bytes ----------------------------------------------------------------
template <class T>
struct Vec;
template <>
struct Vec<__nv_bfloat16> {
  static constexpr int N = 8;
  static constexpr bool kFast = true;
  __device__ static __forceinline__ void unpack(uint4 w, float (&v)[8]) {
    v[0] = bf16_lo(w.x), v[1] = bf16_hi(w.x), v[2] = bf16_lo(w.y), v[3] = bf16_hi(w.y);
    v[4] = bf16_lo(w.z), v[5] = bf16_hi(w.z), v[6] = bf16_lo(w.w), v[7] = bf16_hi(w.w);
  }
  __device__ static __forceinline__ uint4 pack(const float (&v)[8]) {
    return make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]),
                      pack_bf16x2(v[6], v[7]));
  }
};
template <>
struct Vec<float> {
  static constexpr int N = 4;
  static constexpr bool kFast = false;
  __device__ static __forceinline__ void unpack(uint4 w, float (&v)[4]) {
    v[0] = __uint_as_float(w.x), v[1] = __uint_as_float(w.y), v[2] = __uint_as_float(w.z), v[3] = __uint_as_float(w.w);
  }
  __device__ static __forceinline__ uint4 pack(const float (&v)[4]) {
    return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
  }
};

// Calls f with the activation as a constant.
template <class F>
int with_act(int a, F f) {
  switch (a) {
    case LBP_ACT_NONE: return f(std::integral_constant<int, LBP_ACT_NONE>{});
    case LBP_ACT_RELU: return f(std::integral_constant<int, LBP_ACT_RELU>{});
    case LBP_ACT_GELU: return f(std::integral_constant<int, LBP_ACT_GELU>{});
    case LBP_ACT_GELU_TANH: return f(std::integral_constant<int, LBP_ACT_GELU_TANH>{});
    case LBP_ACT_SILU: return f(std::integral_constant<int, LBP_ACT_SILU>{});
  }
  return LBP_ERR_SHAPE;
}

// ---- launchers -----------------------------------------------------------------------------
// Rows of a matrix: element (i, c) at ptr + i * pitch + c.
struct LinearCall {
  const void *x, *W, *bias, *residual;
  void *y, *z;
  long long rows;
  int32_t Cin, Cout, dtype, act;
  int64_t px, pr, py, pz;        // pitches
  int64_t first, step;           // number of element (i, c): first + i * step + c
  Drop drop;
  uint32_t* status;
  void* scratch;
  size_t scratch_bytes;
};
int launch_linear(const LinearCall& c, cudaStream_t stream);
int launch_linear_umma(const LinearCall& c, cudaStream_t stream);   // bf16

// out = residual + drop(a) act'(z) on the tokens of a grid (rows: H = W = 1)
struct PointCall {
  const void *a, *z, *residual;
  void* out;
  long long rows;
  int32_t C, HW, W, dtype, act;
  lbp_view va, vz, vr, vo, number;   // strides
  int64_t first;                     // number of the first element
  Drop drop;
};
int launch_pointwise(const PointCall& c, cudaStream_t stream);

}  // namespace layer
}  // namespace lbp
