// y = residual + drop(act(x W^T + b)): tiles of 64 x 64 on the CUDA cores.
#include "layer_math.cuh"

namespace lbp {
namespace layer {

constexpr int kTile = 64, kDepth = 16;

template <class T, int ACT>
__global__ void __launch_bounds__(256) linear_tile_kernel(const __grid_constant__ LinearCall p) {
  __shared__ float xs[kDepth][kTile + 4], ws[kDepth][kTile + 4];
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const unsigned across = (p.Cout + kTile - 1) / kTile;
  const long long m0 = static_cast<long long>(blockIdx.x / across) * kTile;
  const int n0 = blockIdx.x % across * kTile;
  const T* const x = static_cast<const T*>(p.x);
  const T* const W = static_cast<const T*>(p.W);
  float acc[4][4] = {};
  for (int k0 = 0; k0 < p.Cin; k0 += kDepth) {
    for (int e = threadIdx.x; e < kTile * kDepth; e += 256) {
      const int k = e % kDepth, r = e / kDepth;
      const bool in_k = k0 + k < p.Cin;
      xs[k][r] = in_k && m0 + r < p.rows ? static_cast<float>(x[(m0 + r) * p.px + k0 + k]) : 0.f;
      ws[k][r] = in_k && n0 + r < p.Cout ? static_cast<float>(W[static_cast<long long>(n0 + r) * p.Cin + k0 + k]) : 0.f;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kDepth; ++k) {
      const float4 a = *reinterpret_cast<const float4*>(&xs[k][ty * 4]), b = *reinterpret_cast<const float4*>(&ws[k][tx * 4]);
      const float av[4] = {a.x, a.y, a.z, a.w}, bv[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(av[i], bv[j], acc[i][j]);
    }
    __syncthreads();
  }
  const Stream s = open_stream(p.drop);
  if (blockIdx.x == 0 && threadIdx.x == 0) note_used(p.drop);
  const int c = n0 + tx * 4;
  if (c >= p.Cout) return;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const long long row = m0 + ty * 4 + i;
    if (row >= p.rows) return;
    float v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[j] = acc[i][j];
      if (p.bias != nullptr) v[j] += static_cast<float>(static_cast<const T*>(p.bias)[c + j]);
      if (p.z != nullptr) static_cast<T*>(p.z)[row * p.pz + c + j] = static_cast<T>(v[j]);
      v[j] = act<ACT>(v[j]);
    }
    float out[4] = {};
    if (p.residual != nullptr) {
#pragma unroll
      for (int j = 0; j < 4; ++j) out[j] = static_cast<float>(static_cast<const T*>(p.residual)[row * p.pr + c + j]);
    }
    add_dropped(out, v, p.first + row * p.step + c, s, p.drop);
#pragma unroll
    for (int j = 0; j < 4; ++j) static_cast<T*>(p.y)[row * p.py + c + j] = static_cast<T>(out[j]);
  }
}

static int launch_tile(const LinearCall& c, cudaStream_t stream) {
  const long long tiles = (c.rows + kTile - 1) / kTile;
  return with_act(c.act, [&](auto a) -> int {
    constexpr int ACT = decltype(a)::value;
    const long long grid = tiles * ((c.Cout + kTile - 1) / kTile);
    if (grid >= (1ll << 31)) return LBP_ERR_SHAPE;
    if (c.dtype == LBP_BF16)
      linear_tile_kernel<__nv_bfloat16, ACT><<<static_cast<unsigned>(grid), 256, 0, stream>>>(c);
    else
      linear_tile_kernel<float, ACT><<<static_cast<unsigned>(grid), 256, 0, stream>>>(c);
    count_launch();
    LBP_CUDA_TRY(cudaGetLastError());
    return LBP_OK;
  });
}

int launch_linear(const LinearCall& c, cudaStream_t stream) {
  // coordinates of a tensor map are 32 bits wide
  constexpr long long kMostRows = 1ll << 30;
  LinearCall part = c;
  const int es = c.dtype == LBP_BF16 ? 2 : 4;
  for (long long at = 0; at < c.rows; at += kMostRows) {
    auto from = [&](const void* q, int64_t pitch) { return q == nullptr ? nullptr : static_cast<const uint8_t*>(q) + at * pitch * es; };
    part.rows = c.rows - at < kMostRows ? c.rows - at : kMostRows;
    part.x = from(c.x, c.px);
    part.residual = from(c.residual, c.pr);
    part.y = const_cast<uint8_t*>(from(c.y, c.py));
    part.z = const_cast<uint8_t*>(from(c.z, c.pz));
    part.first = c.first + at * c.step;
    if (int e = c.dtype == LBP_BF16 ? launch_linear_umma(part, stream) : launch_tile(part, stream)) return e;
  }
  return LBP_OK;
}

}  // namespace layer
}  // namespace lbp
