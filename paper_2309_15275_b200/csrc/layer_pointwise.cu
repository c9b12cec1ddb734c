// out = residual + drop(a) act'(z): dropout on its own, and the gradient of a layer's epilogue.
#include "layer_math.cuh"

namespace lbp {
namespace layer {

template <class T, int ACT>
__global__ void __launch_bounds__(256) pointwise_kernel(const __grid_constant__ PointCall p) {
  using V = Vec<T>;
  const Stream s = open_stream(p.drop);
  if (blockIdx.x == 0 && threadIdx.x == 0) note_used(p.drop);
  const int per_row = p.C / V::N;
  const long long n = p.rows * per_row;
  for (long long i = blockIdx.x * 256ll + threadIdx.x; i < n; i += gridDim.x * 256ll) {
    const long long row = i / per_row;
    const int c = static_cast<int>(i - row * per_row) * V::N;
    const long long b = row / p.HW;
    const int t = static_cast<int>(row - b * p.HW), h = t / p.W, w = t - h * p.W;
    auto at = [&](const lbp_view& v) { return b * v.image + h * v.row + w * v.token + c; };
    float v[V::N];
    V::unpack(*reinterpret_cast<const uint4*>(static_cast<const T*>(p.a) + at(p.va)), v);
    if constexpr (ACT != LBP_ACT_NONE) {
      float z[V::N];
      V::unpack(*reinterpret_cast<const uint4*>(static_cast<const T*>(p.z) + at(p.vz)), z);
#pragma unroll
      for (int j = 0; j < V::N; ++j) v[j] *= act_slope<ACT, V::kFast>(z[j]);
    }
    if (p.drop.on) drop(v, p.first + at(p.number), s, p.drop);
    if (p.residual != nullptr) {
      float r[V::N];
      V::unpack(*reinterpret_cast<const uint4*>(static_cast<const T*>(p.residual) + at(p.vr)), r);
#pragma unroll
      for (int j = 0; j < V::N; ++j) v[j] += r[j];
    }
    *reinterpret_cast<uint4*>(static_cast<T*>(p.out) + at(p.vo)) = V::pack(v);
  }
}

int launch_pointwise(const PointCall& c, cudaStream_t stream) {
  const int per_row = c.C / (c.dtype == LBP_BF16 ? 8 : 4);
  const long long n = c.rows * per_row, blocks = (n + 255) / 256;
  const unsigned grid = static_cast<unsigned>(blocks < 148 * 32 ? blocks : 148 * 32);
  return with_act(c.act, [&](auto a) -> int {
    constexpr int ACT = decltype(a)::value;
    if (c.dtype == LBP_BF16)
      pointwise_kernel<__nv_bfloat16, ACT><<<grid, 256, 0, stream>>>(c);
    else
      pointwise_kernel<float, ACT><<<grid, 256, 0, stream>>>(c);
    count_launch();
    LBP_CUDA_TRY(cudaGetLastError());
    return LBP_OK;
  });
}

}  // namespace layer
}  // namespace lbp
