// The elementwise part of a layer's epilogue: activations, their derivatives, and dropout
// from a counter-based generator.
//
// The activations go through the approximate exponential and reciprocal of the special-function unit (2^-22 and 2^-23 of
// their results), two numbers at a time, and polynomials of two lengths: for results that are rounded to bf16, and for fp32
// (FINE).  They take +-infinity to the limit and keep NaN.  What they are off by before that rounding, relative to the result,
// evaluated step by step with an exact exponential and reciprocal (GELU from -13 on, its tanh form from -9.5, SiLU from -86; the
// slopes away from their zeros):
//                    up to -5     -5 .. -2     from -0.5 on    slopes
//   GELU, bf16       4.4e-5       3.7e-5       3.7e-5          7.8e-6, 7.5e-6, 4.7e-5
//   GELU             7.9e-6       1.3e-6       4.3e-7          8.0e-6, 1.3e-6, 7.0e-7
//   tanh form        1.1e-5       2.2e-6       1.8e-7          1.1e-5, 2.3e-6, 2.0e-6
//   SiLU             3.9e-6       3.4e-7       1.6e-7          3.9e-6, 3.9e-7, 9.8e-7
// In the tails that is the exponent u, whose rounding to fp32 moves exp(u) by some |u| 2^-24 of itself.  A reciprocal below
// 2^-126 is 0, so SiLU is from -87.4 on and the tanh form from -10.1 (below 6e-37).
// CUDA's erfcf and expf in their place cost the fp32 gradient of 16384 x 3072 GELUs 107 us, 154 with dropout, instead of 89
// and 97.
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
  uint32_t low15, low_half;   // the same for both halves of a word at once, see kept_halves
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

// Philox4x32-10 (Salmon et al. 2011): the numbers of elements 8 group .. 8 group + 7, two a word, for G
// groups at once, which hides the rounds' latency and shares the key's additions.
template <int G>
__device__ __forceinline__ void philox(const Stream& s, const uint64_t (&group)[G], uint32_t (&w)[4 * G]) {
  uint32_t k0 = s.k0, k1 = s.k1;
  // the round keys are added up here: kept for the next call they would take twenty registers
  asm volatile("" : "+r"(k0), "+r"(k1));
#pragma unroll
  for (int g = 0; g < G; ++g) {
    w[4 * g] = static_cast<uint32_t>(group[g]);
    w[4 * g + 1] = static_cast<uint32_t>(group[g] >> 32);
    w[4 * g + 2] = s.c2;
    w[4 * g + 3] = s.c3;
  }
#pragma unroll
  for (int r = 0; r < 10; ++r) {
#pragma unroll
    for (int g = 0; g < G; ++g) {
      uint32_t* const c = w + 4 * g;
      const uint64_t a = static_cast<uint64_t>(c[0]) * 0xD2511F53u, b = static_cast<uint64_t>(c[2]) * 0xCD9E8D57u;
      c[0] = static_cast<uint32_t>(b >> 32) ^ c[1] ^ k0;
      c[1] = static_cast<uint32_t>(b);
      c[2] = static_cast<uint32_t>(a >> 32) ^ c[3] ^ k1;
      c[3] = static_cast<uint32_t>(a);
    }
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
}
// acc += scale * v where the number in the high half of w is above the bound: a predicated multiply-add,
// which leaves what is dropped out of the sum, whatever it is.
__device__ __forceinline__ void add_kept(float& acc, float v, uint32_t w, const Drop& d) {
  asm("{\n\t.reg .pred p;\n\t"
      "setp.gt.u32 p, %2, %3;\n\t"
      "@p fma.rn.f32 %0, %1, %4, %0;\n\t}"
      : "+f"(acc)
      : "f"(v), "r"(w), "r"(d.above), "f"(d.scale));
}
__device__ __forceinline__ void add_kept2(float& lo, float& hi, float v0, float v1, uint32_t w, const Drop& d) {
  add_kept(lo, v0, w << 16, d);
  add_kept(hi, v1, w, d);
}

// All ones in the halves of w that hold 16-bit numbers u >= t, in four instructions.  With the top bits apart, (u | 2^15) -
// (t mod 2^15) keeps its top bit exactly where u mod 2^15 >= t mod 2^15 and never borrows from the other half; u >= t is
// then "that bit or u's" for t below 2^15, "and" from there on: the majority with low_half.
__device__ __forceinline__ uint32_t kept_halves(uint32_t w, const Drop& d) {
  const uint32_t r = (w | 0x80008000u) - d.low15;
  const uint32_t top = (w & r) | (d.low_half & (w | r));
  uint32_t m;
  asm("prmt.b32 %0, %1, 0, 0xbb99;" : "=r"(m) : "r"(top));   // the sign bits of bytes 1 and 3, all over their halves
  return m;
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

// Two fp32 numbers in a pair of registers: an instruction for both (as long on the FMA pipe, but one issue slot).
struct F2 {
  uint64_t v;
};
__device__ __forceinline__ F2 two(float a, float b) {
  F2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ F2 two(float a) { return two(a, a); }
__device__ __forceinline__ void parts(F2 x, float& a, float& b) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x.v));
}
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) {
  F2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return r;
}
__device__ __forceinline__ F2 mul2(F2 a, F2 b) {
  F2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ F2 add2(F2 a, F2 b) {
  F2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}

// the sign of x, and |x| up to a bound; NaN stays
__device__ __forceinline__ float clamp_abs(float x, float most) {
  float y;
  asm("min.NaN.xorsign.abs.f32 %0, %1, %2;" : "=f"(y) : "f"(x), "f"(most));
  return y;
}

constexpr float kInvSqrt2Pi = 0.3989422804014327f;
constexpr float kLog2e = 1.4426950408889634f;
// 2 sqrt(2/pi) and 0.044715 times that: gelu_tanh(z) = z / (1 + exp(-(A z + B z^3)))
constexpr float kTanhA = 1.5957691216057308f, kTanhB = 0.071354816272600247f;

// The normal distribution's tail Phi(-a), a >= 0, as exp(-a^2/2) Q, with Q = exp(a^2/2) Phi(-a) a polynomial in t = 1 / (1 + c a),
// fitted (weighted least squares towards the smallest largest error): c = 0.38, off by at most 3.7e-5 Q; FINE: c = 0.275,
// 5.1e-8 Q, 3.9e-7 as evaluated.  gelu(z) = max(z, 0) - a Phi(-a), a = |z|.
// a: not above 100 (exp(-a^2/2) is 0 there, and an infinity times that would be NaN).  Hands out exp(-a^2/2) and -Q.
template <bool FINE>
__device__ __forceinline__ void tails(F2 a, F2* e, F2* q) {
  float x, y;
  parts(fma2(a, two(FINE ? 0.275f : 0.38f), two(1.f)), x, y);
  const F2 t = two(rcp(x), rcp(y));
  parts(mul2(a, mul2(a, two(-0.5f * kLog2e))), x, y);
  *e = two(ex2(x), ex2(y));
  F2 p;
  if constexpr (FINE) {
    p = fma2(t, two(-0.027536606416106224f), two(0.11230829358100891f));
    p = fma2(p, t, two(-0.13322971761226654f));
    p = fma2(p, t, two(0.038324955850839615f));
    p = fma2(p, t, two(-0.08998376131057739f));
    p = fma2(p, t, two(-0.07816720008850098f));
    p = fma2(p, t, two(-0.1023753434419632f));
    p = fma2(p, t, two(-0.10962801426649094f));
    p = fma2(p, t, two(-0.10971269756555557f));
    p = fma2(p, t, two(6.223378790082279e-08f));
  } else {
    p = fma2(t, two(0.0906074270606041f), two(-0.1908050775527954f));
    p = fma2(p, t, two(-0.08993600308895111f));
    p = fma2(p, t, two(-0.15882457792758942f));
    p = fma2(p, t, two(-0.15100638568401337f));
    p = fma2(p, t, two(-1.705829163256567e-05f));
  }
  *q = p;
}

// The activation of two numbers.
template <int ACT, bool FINE>
__device__ __forceinline__ void act2(float& z0, float& z1) {
  if constexpr (ACT == LBP_ACT_RELU) {
    z0 = at_least(z0, 0.f);
    z1 = at_least(z1, 0.f);
  } else if constexpr (ACT == LBP_ACT_GELU) {
    // (the factor a makes gelu(0) zero and keeps the error near zero relative; a NaN comes through it)
    const F2 a = two(at_most(fabsf(z0), 100.f), at_most(fabsf(z1), 100.f));
    F2 e, q;
    tails<FINE>(a, &e, &q);
    parts(fma2(a, mul2(e, q), two(fmaxf(z0, 0.f), fmaxf(z1, 0.f))), z0, z1);
  } else if constexpr (ACT == LBP_ACT_GELU_TANH || ACT == LBP_ACT_SILU) {
    // z / (1 + exp(-u))
    constexpr float kLeast = ACT == LBP_ACT_SILU ? -100.f : -30.f;   // (the result is 0 there)
    const F2 c = two(at_least(z0, kLeast), at_least(z1, kLeast));
    F2 u;
    if constexpr (ACT == LBP_ACT_SILU)
      u = mul2(c, two(-kLog2e));
    else
      u = mul2(c, fma2(mul2(c, c), two(-kLog2e * kTanhB), two(-kLog2e * kTanhA)));
    float e0, e1;
    parts(u, e0, e1);
    parts(add2(two(ex2(e0), ex2(e1)), two(1.f)), e0, e1);
    parts(mul2(c, two(rcp(e0), rcp(e1))), z0, z1);
  }
}

// The same where the activation is a call's (uniform) number.
template <bool FINE>
__device__ __forceinline__ void act2_of(int a, float& z0, float& z1) {
  switch (a) {
    case LBP_ACT_RELU: return act2<LBP_ACT_RELU, FINE>(z0, z1);
    case LBP_ACT_GELU: return act2<LBP_ACT_GELU, FINE>(z0, z1);
    case LBP_ACT_GELU_TANH: return act2<LBP_ACT_GELU_TANH, FINE>(z0, z1);
    case LBP_ACT_SILU: return act2<LBP_ACT_SILU, FINE>(z0, z1);
  }
}

// g act'(z) of two numbers.
template <int ACT, bool FINE>
__device__ __forceinline__ void times_slope2(float& g0, float& g1, float z0, float z1) {
  if constexpr (ACT == LBP_ACT_RELU) {
    const float a = at_least(z0, 0.f), b = at_least(z1, 0.f);
    g0 = a > 0.f ? g0 : a;   // (0, or NaN)
    g1 = b > 0.f ? g1 : b;
  } else if constexpr (ACT == LBP_ACT_GELU) {
    // Phi(z) + z phi(z) is h = exp(-a^2/2) (Q - a / sqrt(2 pi)) for z < 0, a = |z|, and 1 - h from zero on.  (Both
    // from 1/2 - h, h would be rounded to a unit of 1/2: 4 % off at -5.5, nothing left at -7.)
    const F2 a = two(at_most(fabsf(z0), 100.f), at_most(fabsf(z1), 100.f));
    F2 e, q;
    tails<FINE>(a, &e, &q);
    const F2 minus_h = mul2(e, fma2(a, two(kInvSqrt2Pi), q));
    float h0, h1, r0, r1;
    parts(minus_h, h0, h1);
    parts(add2(minus_h, two(1.f)), r0, r1);
    parts(mul2(two(g0, g1), two(z0 < 0.f ? -h0 : r0, z1 < 0.f ? -h1 : r1)), g0, g1);
  } else if constexpr (ACT == LBP_ACT_GELU_TANH || ACT == LBP_ACT_SILU) {
    constexpr float kMost = ACT == LBP_ACT_SILU ? 100.f : 12.f;   // (s is 0 and 1 there)
    const F2 c = two(clamp_abs(z0, kMost), clamp_abs(z1, kMost));
    F2 u, v = c;   // the exponent; z u'
    if constexpr (ACT == LBP_ACT_SILU) {
      u = mul2(c, two(-kLog2e));
    } else {
      const F2 c2 = mul2(c, c);
      u = mul2(c, fma2(c2, two(-kLog2e * kTanhB), two(-kLog2e * kTanhA)));
      v = mul2(c, fma2(c2, two(3.f * kTanhB), two(kTanhA)));
    }
    float x, y;
    parts(u, x, y);
    parts(add2(two(ex2(x), ex2(y)), two(1.f)), x, y);
    const F2 s = two(rcp(x), rcp(y));
    // s + v s (1 - s)
    parts(mul2(two(g0, g1), fma2(mul2(v, s), fma2(s, two(-1.f), two(1.f)), s)), g0, g1);
  }
}

// ---- vectors of 16 bytes ----------------------------------------------------------------
template <class T>
struct Vec;
template <>
struct Vec<__nv_bfloat16> {
  static constexpr int N = 8;
  static constexpr bool kFine = false;
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
  static constexpr bool kFine = true;
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

// drop(g) act'(z) of eight bf16 numbers each, where m has all ones in the halves that stay: what is dropped leaves as
// zero, g and z, before any arithmetic.
template <int ACT, bool DROP>
__device__ __forceinline__ void masked_gradient(uint4 g, uint4 z, const uint32_t* m, const Drop& d, float (&v)[8]) {
  using V = Vec<__nv_bfloat16>;
  if constexpr (DROP) g = make_uint4(g.x & m[0], g.y & m[1], g.z & m[2], g.w & m[3]);
  V::unpack(g, v);
  if constexpr (DROP) {
#pragma unroll
    for (int j = 0; j < 8; j += 2) parts(mul2(two(v[j], v[j + 1]), two(d.scale)), v[j], v[j + 1]);
  }
  if constexpr (ACT != LBP_ACT_NONE) {
    float x[8];
    if constexpr (DROP) z = make_uint4(z.x & m[0], z.y & m[1], z.z & m[2], z.w & m[3]);
    V::unpack(z, x);
#pragma unroll
    for (int j = 0; j < 8; j += 2) times_slope2<ACT, false>(v[j], v[j + 1], x[j], x[j + 1]);
  }
}
// drop(g) act'(z) of a vector each of g and z, in fp32: u vectors at once.
template <class T, int ACT, bool DROP, int U>
__device__ __forceinline__ void gradient(const uint4 (&g)[U], const uint4 (&z)[U], const uint64_t (&number)[U], const Stream& s,
                                         const Drop& d, float (&out)[U][Vec<T>::N]) {
  using V = Vec<T>;
  uint32_t w[DROP ? 4 * U : 1];
  if constexpr (DROP) {
    uint64_t group[U];
#pragma unroll
    for (int u = 0; u < U; ++u) group[u] = number[u] >> 3;
    philox<U>(s, group, w);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if constexpr (V::N == 8) {
      uint32_t m[4] = {};
      if constexpr (DROP) {
#pragma unroll
        for (int j = 0; j < 4; ++j) m[j] = kept_halves(w[4 * u + j], d);
      }
      masked_gradient<ACT, DROP>(g[u], z[u], m, d, out[u]);
    } else {
      float v[4];
      V::unpack(g[u], v);
      if constexpr (ACT != LBP_ACT_NONE) {
        float x[4];
        V::unpack(z[u], x);
#pragma unroll
        for (int j = 0; j < 4; j += 2) times_slope2<ACT, true>(v[j], v[j + 1], x[j], x[j + 1]);
      }
      const bool upper = (number[u] & 4u) != 0;
#pragma unroll
      for (int j = 0; j < 4; j += 2) {
        if constexpr (DROP) {
          out[u][j] = out[u][j + 1] = 0.f;
          add_kept2(out[u][j], out[u][j + 1], v[j], v[j + 1], upper ? w[4 * u + 2 + j / 2] : w[4 * u + j / 2], d);
        } else {
          out[u][j] = v[j];
          out[u][j + 1] = v[j + 1];
        }
      }
    }
  }
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
int launch_linear_fp32(const LinearCall& c, cudaStream_t stream);   // (gemm_fp32_split.cu)
// Scratch that a call takes.
size_t linear_scratch_bytes(long long rows, int Cin, int Cout, int dtype);
size_t linear_fp32_scratch_bytes(long long rows, int Cin, int Cout);

// out = residual + drop(a) act'(z) on the tokens of a grid (rows: H = W = 1).  At most one of z and
// residual.
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

// What lbp_project's tensor is formed from where it is a gradient.
struct GradOf {
  const void* z;      // laid out as g_y, or null without an activation
  int32_t act;
  int64_t first;
  lbp_view number;    // resolved
  Drop drop;
};
// Whether the projection kernel of such a call forms the gradient itself.
bool project_forms_gradient(int dtype, int B, int H, int W, int k, int r);
// While set (per calling thread), the first tensor of a projection is what it is formed from.
void set_projection_gradient(const GradOf* of);
const GradOf* projection_gradient();

}  // namespace layer
}  // namespace lbp
