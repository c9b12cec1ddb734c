// out = residual + drop(a) act'(z): dropout on its own, and the gradient of a layer's epilogue.
//
// One pass; a thread has kVectors vectors of 16 bytes of each tensor, 256 threads apart, and asks for all of
// them before it computes.  32768 x 3072 of bf16: GELU's gradient 89 us, 604 MB at 6.8 TB/s; with p = 0.1 118 us
// (28 instructions an element, ten of them for the numbers, in 65 % of the issue slots).
#include "layer_math.cuh"

namespace lbp {
namespace layer {

// Vectors of a thread: with more, more loads are under way and more Philox calls share a key's additions; with
// fewer, more blocks.  32768 x 3072 of bf16 with p = 0.1, 2 / 3 / 4 vectors: GELU's gradient 122 / 120 / 122 us, SiLU's
// 104 / 105 / 101, without an activation 74 / 70 / 68.  (A bound on the registers, for more blocks to an SM, cost 15 %.)
constexpr int kVectors = 3;

// n / d for n < 2^31 without a division: magic numbers from the host (Granlund and Montgomery 1994).
struct Divisor {
  uint32_t d, mul, shift;
};
static Divisor divisor(uint32_t d) {
  uint32_t shift = 0;
  while ((1ull << shift) < d) ++shift;
  return Divisor{d, static_cast<uint32_t>(((1ull << 32) * ((1ull << shift) - d)) / d + 1), shift};
}
__device__ __forceinline__ uint32_t quotient(uint32_t n, const Divisor& v) {
  return static_cast<uint32_t>((static_cast<uint64_t>(__umulhi(n, v.mul)) + n) >> v.shift);
}

struct Grid {
  long long vectors;
  Divisor per_row, HW, W;
};

// FLAT: every tensor, and the numbering, is one run of memory.
template <class T, int ACT, bool DROP, bool FLAT, int U>
__global__ void __launch_bounds__(256) pointwise_kernel(const __grid_constant__ PointCall p, const __grid_constant__ Grid grid) {
  using V = Vec<T>;
  const long long i0 = blockIdx.x * (256ll * U) + threadIdx.x;
  // The kernel ahead may still write what is read here.  (The next one may start when this ends: let in earlier, its
  // blocks take the places of this one's, 11.4 us become 11.9, with lbp_project behind it 16.4 become 17.1.)
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const Stream s = DROP ? open_stream(p.drop) : Stream{};
  if (blockIdx.x == 0 && threadIdx.x == 0) note_used(p.drop);
  uint4 a[U] = {}, z[U] = {};
  uint64_t number[U] = {};
  int64_t out[U];
  const T* const second = static_cast<const T*>(ACT != LBP_ACT_NONE ? p.z : p.residual);
  const lbp_view& v2 = ACT != LBP_ACT_NONE ? p.vz : p.vr;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const long long i = i0 + u * 256;
    if (i >= grid.vectors) break;
    int64_t at, at2;
    if constexpr (FLAT) {
      at = at2 = out[u] = i * V::N;
      number[u] = p.first + at;
    } else {
      long long row, b;
      if (grid.vectors < (1ll << 31)) {
        row = quotient(static_cast<uint32_t>(i), grid.per_row);
        b = quotient(static_cast<uint32_t>(row), grid.HW);
      } else {
        row = i / grid.per_row.d;
        b = row / p.HW;
      }
      const int c = static_cast<int>(i - row * grid.per_row.d) * V::N;
      const uint32_t t = static_cast<uint32_t>(row - b * p.HW), h = quotient(t, grid.W), w = t - h * p.W;
      auto where = [&](const lbp_view& v) { return b * v.image + h * v.row + w * v.token + c; };
      at = where(p.va);
      at2 = second != nullptr ? where(v2) : 0;
      out[u] = where(p.vo);
      number[u] = p.first + where(p.number);
    }
    a[u] = __ldcs(reinterpret_cast<const uint4*>(static_cast<const T*>(p.a) + at));
    if (second != nullptr) z[u] = __ldcs(reinterpret_cast<const uint4*>(second + at2));
  }
  float v[U][V::N];
  gradient<T, ACT, DROP, U>(a, z, number, s, p.drop, v);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (i0 + u * 256 >= grid.vectors) break;
    if (ACT == LBP_ACT_NONE && second != nullptr) {
      float r[V::N];
      V::unpack(z[u], r);
#pragma unroll
      for (int j = 0; j < V::N; ++j) v[u][j] += r[j];
    }
    *reinterpret_cast<uint4*>(static_cast<T*>(p.out) + out[u]) = V::pack(v[u]);
  }
}

int launch_pointwise(const PointCall& call, cudaStream_t stream) {
  PointCall c = call;
  const int N = c.dtype == LBP_BF16 ? 8 : 4;
  const int H = c.HW / c.W;
  // rows that lie one behind the other are one row
  auto one_run = [&](const lbp_view& v) {
    return (c.W == 1 || v.token == c.C) && (H == 1 || v.row == static_cast<int64_t>(c.W) * c.C) &&
           (c.rows == c.HW || v.image == static_cast<int64_t>(c.HW) * c.C);
  };
  const bool flat = one_run(c.va) && one_run(c.vo) && one_run(c.number) && (c.z == nullptr || one_run(c.vz)) &&
                    (c.residual == nullptr || one_run(c.vr));
  Grid g{};
  g.vectors = c.rows * (c.C / N);
  g.per_row = divisor(static_cast<uint32_t>(c.C / N));
  g.HW = divisor(static_cast<uint32_t>(c.HW));
  g.W = divisor(static_cast<uint32_t>(c.W));
  const int per = g.vectors >= 148ll * 2048 * kVectors ? kVectors : 1;   // (all SMs full of threads)
  const long long blocks = (g.vectors + 256ll * per - 1) / (256ll * per);
  if (blocks >= (1ll << 31)) return LBP_ERR_SHAPE;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.gridDim = dim3(static_cast<unsigned>(blocks));
  cfg.blockDim = dim3(256);
  cfg.stream = stream;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return with_act(c.act, [&](auto act) -> int {
    constexpr int ACT = decltype(act)::value;
    auto go = [&](auto t, auto drop, auto f) -> int {
      using T = decltype(t);
      constexpr bool DROP = decltype(drop)::value, FLAT = decltype(f)::value;
      if (per == 1)
        LBP_CUDA_TRY(cudaLaunchKernelEx(&cfg, pointwise_kernel<T, ACT, DROP, FLAT, 1>, c, g));
      else
        LBP_CUDA_TRY(cudaLaunchKernelEx(&cfg, pointwise_kernel<T, ACT, DROP, FLAT, kVectors>, c, g));
      count_launch();
      return LBP_OK;
    };
    auto by_drop = [&](auto t, auto f) -> int {
      return c.drop.on ? go(t, std::true_type{}, f) : go(t, std::false_type{}, f);
    };
    if (c.dtype == LBP_BF16)
      return flat ? by_drop(__nv_bfloat16{}, std::true_type{}) : by_drop(__nv_bfloat16{}, std::false_type{});
    return flat ? by_drop(float{}, std::true_type{}) : by_drop(float{}, std::false_type{});
  });
}

}  // namespace layer
}  // namespace lbp
