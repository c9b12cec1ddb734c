// y = residual + drop(act(x W^T + b)): which kernel a call takes, and those for few tokens.
//
// Few tokens read W once and do next to no arithmetic, so what counts is that every SM has its part of W under way
// at once and that one launch does it all.
//   bf16, up to 16 tokens: a CTA has 16 output channels; its warps take turns on K in steps of 32.  W goes from
//     memory to the registers of mma.sync as its A operand, 16 bytes a lane (lane l: row l / 4 and row l / 4 + 8, k's
//     8 (l % 4) on; the k's of an instruction may come in any order as long as x, the B operand, has the
//     same), so nothing is staged and the tokens cost instructions, not traffic.  The warps' sums meet in shared
//     memory in a fixed order; then a thread has an output.
//   fp32, up to 32 tokens: a warp has two output channels for eight tokens, its lanes run along K, fp32 FMAs.
// 768 -> 3072 channels, one token of bf16: the 4.7 MB of W take 0.7 us from HBM.
#include "layer_math.cuh"
#include "ptx_sm100.cuh"

namespace lbp {
namespace layer {

namespace {

// One element's epilogue, from its product.
template <class T>
__device__ __forceinline__ void finish_one(const LinearCall& p, const Stream& s, long long row, int ch, float v) {
  const T* const bias = static_cast<const T*>(p.bias);
  if (bias != nullptr) v += static_cast<float>(bias[ch]);
  if (p.z != nullptr) static_cast<T*>(p.z)[row * p.pz + ch] = static_cast<T>(v);
  float other = 0.f;
  act2_of<Vec<T>::kFine>(p.act, v, other);
  float out = p.residual != nullptr ? static_cast<float>(static_cast<const T*>(p.residual)[row * p.pr + ch]) : 0.f;
  if (p.drop.on) {
    const uint64_t n = static_cast<uint64_t>(p.first + row * p.step + ch);
    const uint64_t group[1] = {n >> 3};
    uint32_t w[4];
    philox<1>(s, group, w);
    const uint32_t j = static_cast<uint32_t>(n >> 1) & 3u, word = j == 0 ? w[0] : j == 1 ? w[1] : j == 2 ? w[2] : w[3];
    add_kept(out, v, (n & 1u) != 0 ? word : word << 16, p.drop);
  } else {
    out += v;
  }
  static_cast<T*>(p.y)[row * p.py + ch] = static_cast<T>(out);
}

__device__ __forceinline__ void mma_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                          uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// TT: groups of eight tokens; 2^log2_s: CTAs of a cluster, which share K
template <int TT>
__global__ void __launch_bounds__(512) linear_rows_bf16_kernel(const __grid_constant__ LinearCall p, int log2_s) {
  __shared__ float sums[16][16][8 * TT + 1];   // [warp][channel][token]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  const int S = 1 << log2_s, rank = blockIdx.x & (S - 1), group = blockIdx.x >> log2_s;
  const int ch0 = group * 16, r = lane >> 2, c = (lane & 3) * 8;
  const int per = (((p.Cin + 31) / 32 + S - 1) >> log2_s) * 32, k_from = rank * per, k_to = k_from + per < p.Cin ? k_from + per : p.Cin;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const __nv_bfloat16* const W = static_cast<const __nv_bfloat16*>(p.W);
  const __nv_bfloat16* const x = static_cast<const __nv_bfloat16*>(p.x);
  const bool have[2] = {ch0 + r < p.Cout, ch0 + r + 8 < p.Cout};
  float d[TT][4] = {};
  const uint4 none = make_uint4(0u, 0u, 0u, 0u);
  constexpr int U = 4;   // steps under way
  for (int k0 = k_from + warp * 32; k0 < k_to; k0 += warps * 32 * U) {
    uint4 a[U][2], b[U][TT];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = k0 + u * warps * 32 + c;
      const bool in = k < k_to;
#pragma unroll
      for (int h = 0; h < 2; ++h)
        a[u][h] = in && have[h] ? *reinterpret_cast<const uint4*>(W + static_cast<long long>(ch0 + r + 8 * h) * p.Cin + k) : none;
#pragma unroll
      for (int t = 0; t < TT; ++t)
        b[u][t] = in && t * 8 + r < p.rows ? *reinterpret_cast<const uint4*>(x + (t * 8 + r) * p.px + k) : none;
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int t = 0; t < TT; ++t) {
        mma_16816(d[t], a[u][0].x, a[u][1].x, a[u][0].y, a[u][1].y, b[u][t].x, b[u][t].y);
        mma_16816(d[t], a[u][0].z, a[u][1].z, a[u][0].w, a[u][1].w, b[u][t].z, b[u][t].w);
      }
  }
#pragma unroll
  for (int t = 0; t < TT; ++t)
#pragma unroll
    for (int j = 0; j < 4; ++j) sums[warp][r + (j >> 1) * 8][t * 8 + (lane & 3) * 2 + (j & 1)] = d[t][j];
  __syncthreads();
  const Stream s = p.drop.on ? open_stream(p.drop) : Stream{};
  if (blockIdx.x == 0 && threadIdx.x == 0) note_used(p.drop);
  const int outs = 16 * static_cast<int>(p.rows);
  auto sum_of = [&](int e) {
    float v = 0.f;
    for (int w = 0; w < warps; ++w) v += sums[w][e & 15][e >> 4];
    return v;
  };
  auto finish = [&](int e, float v) {
    if (ch0 + (e & 15) < p.Cout) finish_one<__nv_bfloat16>(p, s, e >> 4, ch0 + (e & 15), v);
  };
  if (S == 1) {
    for (int e = threadIdx.x; e < outs; e += blockDim.x) finish(e, sum_of(e));
    return;
  }
  // the CTAs' sums, in the order of their ranks, each output by one of them
  __shared__ float part[16 * 8 * TT];
  for (int e = threadIdx.x; e < outs; e += blockDim.x) part[e] = sum_of(e);
  ptx::cluster_sync_all();
  for (int e = rank * blockDim.x + threadIdx.x; e < outs; e += S * blockDim.x) {
    float v = 0.f;
    for (int q = 0; q < S; ++q) {
      float f;
      asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(f) : "r"(ptx::map_to_rank(ptx::smem_u32(part + e), q)) : "memory");
      v += f;
    }
    finish(e, v);
  }
  ptx::cluster_sync_all();   // no CTA leaves while another may still read its sums
}

__global__ void __launch_bounds__(256) linear_rows_fp32_kernel(const __grid_constant__ LinearCall p) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int ch0 = (blockIdx.x * 8 + warp) * 2;
  const long long t0 = blockIdx.y * 8;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) note_used(p.drop);
  if (ch0 >= p.Cout) return;   // (Cout is a multiple of four: both channels or none)
  const int tokens = p.rows - t0 < 8 ? static_cast<int>(p.rows - t0) : 8;
  const float* const W = static_cast<const float*>(p.W) + static_cast<long long>(ch0) * p.Cin;
  const float* const x = static_cast<const float*>(p.x) + t0 * p.px;
  float sum[2][8] = {};
#pragma unroll 2
  for (int k = lane * 4; k < p.Cin; k += 128) {
    const float4 w0 = *reinterpret_cast<const float4*>(W + k), w1 = *reinterpret_cast<const float4*>(W + p.Cin + k);
#pragma unroll
    for (int t = 0; t < 8; ++t) {
      if (t < tokens) {
        const float4 v = *reinterpret_cast<const float4*>(x + t * p.px + k);
        sum[0][t] = fmaf(w0.w, v.w, fmaf(w0.z, v.z, fmaf(w0.y, v.y, fmaf(w0.x, v.x, sum[0][t]))));
        sum[1][t] = fmaf(w1.w, v.w, fmaf(w1.z, v.z, fmaf(w1.y, v.y, fmaf(w1.x, v.x, sum[1][t]))));
      }
    }
  }
  // lane l ends up with output l of the sixteen (channel l / 8, token l % 8): halves of the lanes keep halves of the outputs
  float v[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] = sum[i >> 3][i & 7];
#pragma unroll
  for (int n = 8; n >= 1; n >>= 1) {
#pragma unroll
    for (int i = 0; i < n; ++i) {
      const bool up = (lane & n) != 0;
      const float keep = up ? v[i + n] : v[i], give = up ? v[i] : v[i + n];
      v[i] = keep + __shfl_xor_sync(0xffffffffu, give, n);
    }
  }
  v[0] += __shfl_xor_sync(0xffffffffu, v[0], 16);
  const int t = lane & 7;
  if (lane >= 16 || t >= tokens) return;
  const Stream s = p.drop.on ? open_stream(p.drop) : Stream{};
  finish_one<float>(p, s, t0 + t, ch0 + (lane >> 3), v[0]);
}

template <class Kernel, class... More>
int launch(Kernel kernel, dim3 grid, int threads, int cluster, cudaStream_t stream, More... more) {
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  LBP_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, more...));
  count_launch();
  return LBP_OK;
}

int launch_rows(const LinearCall& c, cudaStream_t stream) {
  if (c.dtype == LBP_F32)
    return launch(linear_rows_fp32_kernel, dim3((c.Cout + 15) / 16, (c.rows + 7) / 8), 256, 1, stream, c);
  // CTAs for all SMs, as long as each has 256 k's and more; a warp for every 32 of them
  const int groups = (c.Cout + 15) / 16;
  int log2_s = 0;
  while (log2_s < 3 && (groups << (log2_s + 1)) <= 296 && (c.Cin >> (log2_s + 1)) >= 256) ++log2_s;
  const int S = 1 << log2_s, steps = ((c.Cin + 31) / 32 + S - 1) / S, warps = steps < 4 ? 4 : steps < 16 ? steps : 16;
  if (c.rows <= 8) return launch(linear_rows_bf16_kernel<1>, dim3(groups * S), warps * 32, S, stream, c, log2_s);
  return launch(linear_rows_bf16_kernel<2>, dim3(groups * S), warps * 32, S, stream, c, log2_s);
}

// Tokens that count as few.
int few_tokens(int dtype) { return dtype == LBP_F32 ? 32 : 16; }

}  // namespace

size_t linear_scratch_bytes(long long rows, int Cin, int Cout, int dtype) {
  if (rows <= few_tokens(dtype)) return 0;
  return dtype == LBP_F32 ? linear_fp32_scratch_bytes(rows, Cin, Cout) : 0;
}

int launch_linear(const LinearCall& c, cudaStream_t stream) {
  if (c.rows <= few_tokens(c.dtype)) return launch_rows(c, stream);
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
    if (int e = c.dtype == LBP_BF16 ? launch_linear_umma(part, stream) : launch_linear_fp32(part, stream)) return e;
  }
  return LBP_OK;
}

}  // namespace layer
}  // namespace lbp
