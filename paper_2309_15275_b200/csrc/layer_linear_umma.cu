// y = residual + drop(act(x W^T + b)) for bf16 data on the tcgen05 tensor cores, the whole epilogue
// behind the accumulator.
//
// A tile is 128 tokens by BN output channels; both operands are K-major as they lie (x by tokens, W by
// output channels).  On CTA pairs (cta_group::2) a tile is 256 tokens, and each CTA fetches its own 128
// tokens and half of W's rows.  Persistent, two accumulators in TMEM, so that the epilogue of a tile runs
// under the products of the next.  Tiles go to the units round robin, a token tile's columns
// next to one another, so that x comes from HBM once and W stays in L2.
//
// Warps: 0 TMA loads, 1 tcgen05, 2-17 the epilogue, four to each quarter of the accumulator's lanes, which
// take turns on its chunks of 64 columns.  Such a warp works alone on its 32 tokens x 64 channels, 16 channels at a
// time.  A thread has a token, so that its channels lie together and one Philox call serves eight of them.  The
// results go to a box in shared memory and out by TMA, which clips what hangs over the last token and channel: y of 64
// channels, or z and y of 32.  The residual is read 32 bytes (a sector) a thread.
//
// What bounds it, at 32768 tokens 768 -> 3072 and 1965 MHz: the operands' way from L2 (1.2 GB: 93 us without any
// store, 1.66 PFLOP/s), which the stores share (y 116, z too 140), and with GELU and dropout the epilogue's arithmetic
// (27 instructions an element; 163); long runs the power cap (189 at 1.4 GHz).  200704 tokens 48 -> 192, one k-block a tile: 28
// us without an activation, 36 with GELU.  Tried before the arithmetic was what it is now, against 116, 144 and 171 us: a 32-byte store a thread without shared memory (112, 149, 175, and 48 -> 192
// channels 46 instead of 43), a bulk copy per row by its thread (116, 201, 297), twelve warps (116, 142, 185).  z
// in a pass of its own, against 135 and 151: 139 and 155, 48 -> 192 channels 40 instead of 37, GELU without dropout 134 instead of 138.
#include "layer_math.cuh"
#include "ptx_sm100.cuh"

namespace lbp {
namespace layer {

namespace {

constexpr int kBM = 128, kBK = 64;
constexpr int kABytes = kBM * kBK * 2;
constexpr int kPerQuarter = 4, kEpilogueWarps = 4 * kPerQuarter;
constexpr int kThreads = (2 + kEpilogueWarps) * 32;
constexpr int kBoxBytes = 32 * 128;
constexpr int kBiasBytes = 2 * kPerQuarter * 64 * 4, kOutBytes = kEpilogueWarps * kBoxBytes;   // bias: of a tile and the next
constexpr int kMaxStages = 8;
constexpr int kBarBytes = 256;
constexpr int kSmemMax = 227 * 1024;
constexpr uint32_t kTmemCols = 512, kSlotCols = 256;
constexpr uint32_t kSite = 8u << 16;

struct Params {
  const __nv_bfloat16 *bias, *residual;
  __nv_bfloat16 *y, *z;
  long long rows;
  int64_t pr, py, pz;
  int32_t Cout, BN, num_kb, tiles_n, tiles, stages, stage_bytes;
  int32_t wide, test_stall;   // rows of y, z and the residual start on 32-byte boundaries
  int64_t first, step;
  Drop drop;
  uint32_t* status;
};
struct Maps {
  CUtensorMap x, W, y, z;
};

__device__ __forceinline__ void store_2d(const CUtensorMap* m, const void* src, int32_t x, int32_t y) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];" ::"l"(
                   reinterpret_cast<uint64_t>(m)),
               "r"(ptx::smem_u32(src)), "r"(x), "r"(y)
               : "memory");
}
// 16 channels of a row, as far as they go (`n` of them).
__device__ __forceinline__ void write16(__nv_bfloat16* to, const uint32_t (&w)[8], int n, bool wide) {
  if (wide && n >= 16) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(w[0]), "r"(w[1]), "r"(w[2]),
                 "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                 : "memory");
  } else {
    if (n > 0) *reinterpret_cast<uint4*>(to) = make_uint4(w[0], w[1], w[2], w[3]);
    if (n > 8) *reinterpret_cast<uint4*>(to + 8) = make_uint4(w[4], w[5], w[6], w[7]);
  }
}
__device__ __forceinline__ void bulk_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
__device__ __forceinline__ void bulk_wait_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
__device__ __forceinline__ void bulk_wait_all() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
__device__ __forceinline__ void read16(const __nv_bfloat16* from, uint32_t (&w)[8], int n, bool wide) {
  if (wide && n >= 16) {
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                 : "l"(from)
                 : "memory");
  } else {
    uint4 a = make_uint4(0u, 0u, 0u, 0u), b = a;
    if (n > 0) a = *reinterpret_cast<const uint4*>(from);
    if (n > 8) b = *reinterpret_cast<const uint4*>(from + 8);
    w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w, w[4] = b.x, w[5] = b.y, w[6] = b.z, w[7] = b.w;
  }
}

// Row and column of a unit's tiles, one after the other.
struct Walk {
  int m, n, step_m, step_n;
  __device__ __forceinline__ Walk(const Params& p, int unit, int units) {
    m = unit / p.tiles_n, n = unit - m * p.tiles_n;
    step_m = units / p.tiles_n, step_n = units - step_m * p.tiles_n;
  }
  __device__ __forceinline__ void advance(const Params& p) {
    m += step_m;
    n += step_n;
    if (n >= p.tiles_n) {
      n -= p.tiles_n;
      ++m;
    }
  }
};

// After an expired wait, one thread: the MMAs of the first `mmas` blocks and the loads of the first `loads` have ended, or
// another wait has run out, before memory that they touch is given back.  (Earlier uses of a stage have ended: its later
// ones waited for them.)
__device__ __forceinline__ void settle(uint64_t* full, uint64_t* empty, int stages, int loads, int mmas, uint32_t* status) {
  if (mmas > 0) ptx::mbar_wait_parked(&empty[(mmas - 1) % stages], ((mmas - 1) / stages) & 1u, status, kSite | 5u);
  for (int u = loads > stages ? loads - stages : 0; u < loads; ++u)
    if (!ptx::mbar_wait_parked(&full[u % stages], (u / stages) & 1u, status, kSite | 6u)) return;
}
__device__ __forceinline__ void store_cluster(uint32_t addr, int v) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}
// Blocks that are fetched while a test stalls the loads (0: it does not).
__device__ __forceinline__ int most_loads(int test_stall) { return test_stall == 0 ? 0x7fffffff : test_stall - 1; }

template <int ACT, bool DROP, bool RES, bool ZY, bool PAIR>
__global__ void __launch_bounds__(kThreads, 1)
    linear_umma_kernel(const __grid_constant__ Maps tm, const __grid_constant__ Params p) {
  constexpr int kCtas = PAIR ? 2 : 1;
  extern __shared__ __align__(1024) uint8_t smem[];
  uint8_t* const outs = smem + p.stages * p.stage_bytes;
  float* const biases = reinterpret_cast<float*>(outs + kOutBytes);
  uint64_t* const full = reinterpret_cast<uint64_t*>(reinterpret_cast<uint8_t*>(biases) + kBiasBytes);   // [kMaxStages]
  uint64_t* const empty = full + kMaxStages;
  uint64_t* const acc_full = empty + kMaxStages;    // [2]
  uint64_t* const acc_empty = acc_full + 2;         // [2], the leader's are used
  uint32_t* const tmem_slot = reinterpret_cast<uint32_t*>(acc_empty + 2);
  volatile int* const abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  volatile int* const counts = abort_flag + 1;      // [3]: blocks loaded by the leader, by its peer; blocks multiplied

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = PAIR ? static_cast<int>(ptx::cluster_ctarank()) : 0;
  const int unit = blockIdx.x / kCtas, units = gridDim.x / kCtas;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kMaxStages; ++s) {
      ptx::mbar_init(&full[s], 1);
      ptx::mbar_init(&empty[s], 1);
    }
    for (int s = 0; s < 2; ++s) {
      ptx::mbar_init(&acc_full[s], 1);
      ptx::mbar_init(&acc_empty[s], kCtas * kEpilogueWarps);
    }
    ptx::mbar_fence_init();
    *abort_flag = 0;
    counts[0] = counts[1] = counts[2] = 0;
    ptx::prefetch_tensormap(&tm.x);
    ptx::prefetch_tensormap(&tm.W);
  }
  if (warp == 1) {
    if constexpr (PAIR) {
      ptx::tmem_alloc_pair(tmem_slot, kTmemCols);
      ptx::tmem_relinquish_pair();
    } else {
      ptx::tmem_alloc(tmem_slot, kTmemCols);
      ptx::tmem_relinquish();
    }
  }
  ptx::tc_fence_before_sync();
  __syncthreads();
  if constexpr (PAIR) ptx::cluster_sync_all();
  ptx::tc_fence_after_sync();
  const uint32_t tmem_base = *tmem_slot;
  // nothing is read or written before the kernel ahead has completed
  asm volatile("griddepcontrol.wait;" ::: "memory");

  if (warp == 0) {
    // =========================== loads ===========================
    if (ptx::elect_one()) {
      asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
      const uint64_t keep = ptx::l2_policy_evict_last();
      const int part = p.BN / kCtas;   // W's rows of this CTA
      const uint32_t tx = static_cast<uint32_t>(kCtas * (kABytes + part * kBK * 2));
      int s = 0, loads = 0;
      uint32_t phase = 0;
      bool ok = true;
      const int most = most_loads(p.test_stall);
      Walk at(p, unit, units);
      for (int t = unit; t < p.tiles && ok && loads < most; t += units, at.advance(p)) {
        const int row = (at.m * kCtas + rank) * kBM, col = at.n * p.BN + rank * part;
        for (int kb = 0; kb < p.num_kb && loads < most; ++kb) {
          if (!ptx::mbar_wait_parked(&empty[s], phase ^ 1u, p.status, kSite | 1u)) {
            ok = false;
            break;
          }
          uint8_t* const sa = smem + s * p.stage_bytes;
          if (rank == 0) ptx::mbar_expect_tx(&full[s], tx);   // boxes count in full, also where they hang over
          if constexpr (PAIR) {
            const uint32_t bar = ptx::map_to_rank(ptx::smem_u32(&full[s]), 0);
            ptx::tma_load_2d_pair(sa, &tm.x, bar, kb * kBK, row, keep);
            ptx::tma_load_2d_pair(sa + kABytes, &tm.W, bar, kb * kBK, col, keep);
          } else {
            ptx::tma_load_2d_hint(sa, &tm.x, &full[s], kb * kBK, row, keep);
            ptx::tma_load_2d_hint(sa + kABytes, &tm.W, &full[s], kb * kBK, col, keep);
          }
          ++loads;
          if (++s == p.stages) {
            s = 0;
            phase ^= 1u;
          }
        }
      }
      if (PAIR && rank != 0)
        store_cluster(ptx::map_to_rank(ptx::smem_u32(const_cast<int*>(counts + 1)), 0), loads);
      else
        counts[0] = loads;
      if (!ok) *abort_flag = 1;
    }
  } else if (warp == 1) {
    // =========================== tcgen05 (leader only) ===========================
    if (rank == 0 && ptx::elect_one()) {
      const uint32_t idesc = ptx::idesc_bf16(kCtas * kBM, p.BN, false, false);
      auto commit = [](uint64_t* bar) {
        if constexpr (PAIR)
          ptx::mma_commit_pair(bar);
        else
          ptx::mma_commit(bar);
      };
      int s = 0, n = 0, mmas = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int t = unit; t < p.tiles && ok; t += units, ++n) {
        const uint32_t d = tmem_base + (n & 1) * kSlotCols;
        if (!ptx::mbar_wait_parked(&acc_empty[n & 1], ((n >> 1) + 1) & 1u, p.status, kSite | 2u)) {
          ok = false;
          break;
        }
        for (int kb = 0; kb < p.num_kb; ++kb) {
          if (!ptx::mbar_wait_parked(&full[s], phase, p.status, kSite | 3u)) {
            ok = false;
            break;
          }
          ptx::tc_fence_after_sync();
          const uint32_t sa = ptx::smem_u32(smem + s * p.stage_bytes), sb = sa + kABytes;
#pragma unroll
          for (int kk = 0; kk < kBK / 16; ++kk) {
            const uint64_t da = ptx::smem_desc_sw128(sa + kk * 32, 16, 1024), db = ptx::smem_desc_sw128(sb + kk * 32, 16, 1024);
            const uint32_t add = (kb == 0 && kk == 0) ? 0u : 1u;
            if constexpr (PAIR)
              ptx::mma_bf16_ss_pair(d, da, db, idesc, add);
            else
              ptx::mma_bf16_ss(d, da, db, idesc, add);
          }
          commit(&empty[s]);
          ++mmas;
          if (++s == p.stages) {
            s = 0;
            phase ^= 1u;
          }
        }
        if (ok) commit(&acc_full[n & 1]);
      }
      counts[2] = mmas;
      if (!ok) *abort_flag = 1;
    }
  } else {
    // =========================== epilogue ===========================
    const int e = warp - 2, quarter = warp & 3;
    uint8_t* const box = outs + e * kBoxBytes;
    const Stream stream = DROP ? open_stream(p.drop) : Stream{};
    if (blockIdx.x == 0 && warp == 2 && lane == 0) note_used(p.drop);
    const int chunks = p.BN / 64;
    bool ok = true;
    int n = 0, next = e >> 2;   // chunks go round, so that every warp has as many
    Walk at(p, unit, units);
    for (int t = unit; t < p.tiles && ok; t += units, ++n, at.advance(p)) {
      const int m = at.m;
      const long long row = static_cast<long long>(m * kCtas + rank) * kBM + quarter * 32 + lane;
      bool waited = false;
      auto wait = [&] {
        waited = true;
        ok = __all_sync(0xffffffffu, ptx::mbar_wait_parked(&acc_full[n & 1], static_cast<uint32_t>(n >> 1) & 1u, p.status, kSite | 4u) &&
                                         *abort_flag == 0);
        ptx::tc_fence_after_sync();
      };
      int c = next;
      static_assert(kPerQuarter >= 4, "at most one chunk of a tile a warp: the biases of a tile are written once");
      for (; c < chunks; c += kPerQuarter) {
        const int col = at.n * p.BN + c * 64;
        const int cols = p.Cout - col;                           // of this chunk on
        const int here = row < p.rows ? cols : 0;                // ... in this thread's row
        const uint32_t two_biases = p.bias != nullptr && 2 * lane < cols ? *(reinterpret_cast<const uint32_t*>(p.bias + col) + lane) : 0u;
        const __nv_bfloat16* const res = p.residual + row * p.pr + col;
        uint32_t r[8];
        if constexpr (RES) read16(res, r, here, p.wide);
        if (!waited) wait();
        if (!ok) break;
        // The four warps of these columns write the same.  (What is overwritten belongs to the tile before the last,
        // whose accumulator every warp has released.)
        float* const bias = biases + ((n & 1) * kPerQuarter + (e >> 2)) * 64;
        *reinterpret_cast<float2*>(bias + 2 * lane) = make_float2(bf16_lo(two_biases), bf16_hi(two_biases));
        __syncwarp();
        const uint32_t acc = tmem_base + (static_cast<uint32_t>(quarter * 32) << 16) + (n & 1) * kSlotCols + c * 64;
        const uint64_t number = static_cast<uint64_t>(p.first + row * p.step + col);
        // y of 64 channels takes the whole box, in the 128-byte swizzle; z and y of 32 a half each, in the 64-byte one
        auto put = [&](bool first_half, int h, const uint32_t (&w)[8]) {
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            uint8_t* const to = ZY ? box + (first_half ? 0 : kBoxBytes / 2) + lane * 64 + ((((h & 1) * 2 + g) ^ ((lane >> 1) & 3)) << 4)
                                   : box + lane * 128 + (((h * 2 + g) ^ (lane & 7)) << 4);
            *reinterpret_cast<uint4*>(to) = make_uint4(w[4 * g], w[4 * g + 1], w[4 * g + 2], w[4 * g + 3]);
          }
        };
        // 16 channels at h * 16, from the accumulator in a
        auto step = [&](int h, const uint32_t (&a)[16]) {
          float v[16], out[16];
#pragma unroll
          for (int j = 0; j < 16; ++j) v[j] = __uint_as_float(a[j]);
#pragma unroll
          for (int j = 0; j < 16; j += 4) {   // (zeros without a bias)
            const float4 b = *reinterpret_cast<const float4*>(bias + h * 16 + j);
            parts(add2(two(v[j], v[j + 1]), two(b.x, b.y)), v[j], v[j + 1]);
            parts(add2(two(v[j + 2], v[j + 3]), two(b.z, b.w)), v[j + 2], v[j + 3]);
          }
          const int left = here - h * 16;
          uint32_t w[8];
          uint32_t zw[8];
          if constexpr (ZY) {
#pragma unroll
            for (int j = 0; j < 8; ++j) zw[j] = pack_bf16x2(v[2 * j], v[2 * j + 1]);
          }
#pragma unroll
          for (int j = 0; j < 16; j += 2) act2<ACT, false>(v[j], v[j + 1]);
          if constexpr (RES) {
#pragma unroll
            for (int j = 0; j < 8; ++j) out[2 * j] = bf16_lo(r[j]), out[2 * j + 1] = bf16_hi(r[j]);
            if (h < 3) read16(res + (h + 1) * 16, r, left - 16, p.wide);
          }
          if constexpr (DROP) {
            const uint64_t g0 = (number >> 3) + h * 2, group[2] = {g0, g0 + 1};
            philox<2>(stream, group, w);
          }
          if constexpr (DROP && !RES) {   // what is dropped is cleared in the packed result
#pragma unroll
            for (int j = 0; j < 16; j += 2) parts(mul2(two(v[j], v[j + 1]), two(p.drop.scale)), v[j], v[j + 1]);
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = pack_bf16x2(v[2 * j], v[2 * j + 1]) & kept_halves(w[j], p.drop);
          } else {
            if constexpr (DROP) {
#pragma unroll
              for (int j = 0; j < 8; ++j) add_kept2(out[2 * j], out[2 * j + 1], v[2 * j], v[2 * j + 1], w[j], p.drop);
            } else if constexpr (RES) {
#pragma unroll
              for (int j = 0; j < 16; j += 2) parts(add2(two(out[j], out[j + 1]), two(v[j], v[j + 1])), out[j], out[j + 1]);
            } else {
#pragma unroll
              for (int j = 0; j < 16; ++j) out[j] = v[j];
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = pack_bf16x2(out[2 * j], out[2 * j + 1]);
          }
          if (h == 0 || (ZY && h == 2)) {
            if (lane == 0) bulk_wait_read();   // what the box held has been sent
            __syncwarp();
          }
          if constexpr (ZY) put(true, h, zw);
          put(false, h, w);
          if constexpr (RES) __syncwarp();   // (rows past the last read nothing: together again for the accumulator)
        };
        auto send = [&](int from) {   // the box, whose channels begin `from` further on
          ptx::fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) {
            if (col + from < p.Cout && row < p.rows) {
              if constexpr (ZY) store_2d(&tm.z, box, col + from, static_cast<int32_t>(row));
              store_2d(&tm.y, ZY ? box + kBoxBytes / 2 : box, col + from, static_cast<int32_t>(row));
            }
            bulk_commit();
          }
          __syncwarp();   // what follows reads the accumulator, with all lanes at once
        };
        uint32_t a0[16];
        if constexpr (DROP && RES) {   // (the registers are needed otherwise)
#pragma unroll 1
          for (int h = 0; h < 4; ++h) {
            ptx::tmem_ld_32x16(acc + h * 16, a0);
            ptx::tmem_ld_wait();
            step(h, a0);
            if (ZY && h == 1) send(0);
          }
        } else {   // a step's accumulator is read while the one before is worked on
          uint32_t a1[16];
          ptx::tmem_ld_32x16(acc, a0);
          ptx::tmem_ld_wait();
#pragma unroll 1
          for (int h = 0; h < 4; h += 2) {
            ptx::tmem_ld_32x16(acc + (h + 1) * 16, a1);
            step(h, a0);
            ptx::tmem_ld_wait();
            if (h == 0) ptx::tmem_ld_32x16(acc + 32, a0);
            step(h + 1, a1);
            ptx::tmem_ld_wait();
            if (ZY && h == 0) send(0);
          }
        }
        send(ZY ? 32 : 0);
      }
      next = c - chunks;
      if (!waited) wait();
      // the accumulator has been read
      ptx::tc_fence_before_sync();
      __syncwarp();
      if (lane == 0 && ok) {
        if constexpr (PAIR)
          ptx::mbar_arrive_cluster(ptx::map_to_rank(ptx::smem_u32(&acc_empty[n & 1]), 0));
        else
          ptx::mbar_arrive(&acc_empty[n & 1]);
      }
    }
    if (!ok && lane == 0) *abort_flag = 1;
    bulk_wait_all();   // everything has been written before the CTA leaves
  }

  ptx::tc_fence_before_sync();
  __syncthreads();
  if constexpr (PAIR) {
    if (threadIdx.x == 0 && *abort_flag != 0)
      store_cluster(ptx::map_to_rank(ptx::smem_u32(const_cast<int*>(abort_flag)), rank ^ 1), 1);
    ptx::cluster_sync_all();   // neither CTA leaves while the other may still touch its memory
  }
  if (*abort_flag != 0) {   // (the same in both CTAs; the pair's loads and MMAs signal on the leader's barriers)
    if (rank == 0 && threadIdx.x == 0)
      settle(full, empty, p.stages, counts[0] > counts[1] ? counts[0] : counts[1], counts[2], p.status);
    __syncthreads();
    if constexpr (PAIR) ptx::cluster_sync_all();
  }
  if (warp == 1) {
    ptx::tc_fence_after_sync();
    if constexpr (PAIR)
      ptx::tmem_dealloc_pair(tmem_base, kTmemCols);
    else
      ptx::tmem_dealloc(tmem_base, kTmemCols);
  }
}

// ---- few tiles: K shared among the CTAs of a cluster ----
//
// Where the tiles leave SMs without one, the S CTAs of a cluster take a tile together, each a run of its k-blocks.  Their
// accumulators go to shared memory, and after a cluster barrier CTA r adds up, in the order of the ranks, its share of
// the columns, 16 at a time, from all of them (distributed shared memory) and runs the epilogue on those: one launch,
// no planes, sums in a fixed order.  An SM gets 60 bytes a cycle of operands, so what counts is a CTA's bytes, and
// tiles of 128 columns with more CTAs to a tile beat 64 (1024 tokens 3072 -> 768: 12.4 us unshared).
constexpr int kSplitStages = 6;
constexpr int kSplitThreads = 10 * 32;
constexpr int kSplitSmem = kSplitStages * (kABytes + 128 * kBK * 2) + kBarBytes;
static_assert(kBM * 128 * 4 <= kSplitStages * kABytes, "the sums take the operands' place");

__device__ __forceinline__ float4 ld_cluster(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
  return v;
}

template <int ACT, bool DROP, int S>
__global__ void __launch_bounds__(kSplitThreads, 1)
    linear_split_kernel(const __grid_constant__ Maps tm, const __grid_constant__ Params p) {
  extern __shared__ __align__(1024) uint8_t smem[];
  const int stage_bytes = p.stage_bytes, BN = p.BN;
  uint64_t* const full = reinterpret_cast<uint64_t*>(smem + kSplitStages * stage_bytes);
  uint64_t* const empty = full + kSplitStages;
  uint64_t* const acc_full = empty + kSplitStages;
  uint32_t* const tmem_slot = reinterpret_cast<uint32_t*>(acc_full + 1);
  volatile int* const abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  volatile int* const counts = abort_flag + 1;   // [2]: blocks loaded, multiplied
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = static_cast<int>(ptx::cluster_ctarank()), tile = blockIdx.x / S;
  const int m = tile / p.tiles_n, col0 = (tile - m * p.tiles_n) * BN;
  const int per = (p.num_kb + S - 1) / S, kb0 = rank * per, kb1 = kb0 + per < p.num_kb ? kb0 + per : p.num_kb;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kSplitStages; ++s) {
      ptx::mbar_init(&full[s], 1);
      ptx::mbar_init(&empty[s], 1);
    }
    ptx::mbar_init(acc_full, 1);
    ptx::mbar_fence_init();
    *abort_flag = counts[0] = counts[1] = 0;
    ptx::prefetch_tensormap(&tm.x);
    ptx::prefetch_tensormap(&tm.W);
  }
  if (warp == 1) {
    ptx::tmem_alloc(tmem_slot, BN);
    ptx::tmem_relinquish();
  }
  ptx::tc_fence_before_sync();
  __syncthreads();
  ptx::tc_fence_after_sync();
  const uint32_t tmem_base = *tmem_slot;
  asm volatile("griddepcontrol.wait;" ::: "memory");

  if (warp == 0) {
    if (ptx::elect_one()) {
      asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
      const uint64_t keep = ptx::l2_policy_evict_last();
      const int most = most_loads(p.test_stall);
      int i = 0;
      for (int kb = kb0; kb < kb1 && i < most; ++kb, ++i) {
        const int s = i % kSplitStages;
        if (!ptx::mbar_wait_parked(&empty[s], ((i / kSplitStages) + 1) & 1u, p.status, kSite | 7u)) {
          *abort_flag = 1;
          break;
        }
        uint8_t* const sa = smem + s * stage_bytes;
        ptx::mbar_expect_tx(&full[s], stage_bytes);
        ptx::tma_load_2d_hint(sa, &tm.x, &full[s], kb * kBK, m * kBM, keep);
        ptx::tma_load_2d_hint(sa + kABytes, &tm.W, &full[s], kb * kBK, col0, keep);
      }
      counts[0] = i;
    }
  } else if (warp == 1) {
    if (ptx::elect_one()) {
      const uint32_t idesc = ptx::idesc_bf16(kBM, BN, false, false);
      bool ok = true;
      int i = 0;
      for (int kb = kb0; kb < kb1; ++kb, ++i) {
        const int s = i % kSplitStages;
        ok = ptx::mbar_wait_parked(&full[s], (i / kSplitStages) & 1u, p.status, kSite | 8u);
        if (!ok) break;
        ptx::tc_fence_after_sync();
        const uint32_t sa = ptx::smem_u32(smem + s * stage_bytes), sb = sa + kABytes;
#pragma unroll
        for (int kk = 0; kk < kBK / 16; ++kk)
          ptx::mma_bf16_ss(tmem_base, ptx::smem_desc_sw128(sa + kk * 32, 16, 1024), ptx::smem_desc_sw128(sb + kk * 32, 16, 1024),
                           idesc, (i == 0 && kk == 0) ? 0u : 1u);
        ptx::mma_commit(&empty[s]);
      }
      counts[1] = i;
      if (ok)
        ptx::mma_commit(acc_full);
      else
        *abort_flag = 1;
    }
  }
  const int quarter = warp & 3, row = quarter * 32 + lane, half = (warp - 2) >> 2;   // warps 2-9: a row of the tile a thread, every other 16 columns
  float* const part = reinterpret_cast<float*>(smem);        // four columns of a row at ((column / 4) * 128 + row) * 4
  if (warp >= 2) {
    // (a CTA without k-blocks, where they do not share out evenly, has zeros)
    bool ok = kb0 < kb1;
    if (ok) {
      ok = __all_sync(0xffffffffu, ptx::mbar_wait_parked(acc_full, 0, p.status, kSite | 9u));
      if (!ok) *abort_flag = 1;
    }
    ptx::tc_fence_after_sync();
#pragma unroll 1
    for (int c = half * 16; c < BN; c += 32) {
      uint32_t a[16];
      if (ok) {
        ptx::tmem_ld_32x16(tmem_base + (static_cast<uint32_t>(quarter * 32) << 16) + c, a);
        ptx::tmem_ld_wait();
      } else {
#pragma unroll
        for (int j = 0; j < 16; ++j) a[j] = 0u;
      }
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *reinterpret_cast<uint4*>(part + ((c / 4 + j) * kBM + row) * 4) = make_uint4(a[4 * j], a[4 * j + 1], a[4 * j + 2], a[4 * j + 3]);
    }
  }
  ptx::tc_fence_before_sync();
  __syncthreads();
  if (*abort_flag != 0) {
    if (threadIdx.x == 0) settle(full, empty, kSplitStages, counts[0], counts[1], p.status);
    __syncthreads();
  }
  ptx::cluster_sync_all();
  if (warp == 1) {
    ptx::tc_fence_after_sync();
    ptx::tmem_dealloc(tmem_base, BN);
  }
  if (warp >= 2) {
    const Stream stream = DROP ? open_stream(p.drop) : Stream{};
    if (blockIdx.x == 0 && threadIdx.x == 64) note_used(p.drop);
    const long long grow = static_cast<long long>(m) * kBM + row;
    const int steps = BN / 16, to = (rank + 1) * steps / S * 16;
#pragma unroll 1
    for (int c = (rank * steps / S + half) * 16; c < to; c += 32) {
      const int col = col0 + c, left = grow < p.rows ? p.Cout - col : 0;
      float v[16], out[16];
      uint32_t w[8];
#pragma unroll
      for (int j = 0; j < 16; ++j) out[j] = 0.f;
      if (p.residual != nullptr) {
        read16(p.residual + grow * p.pr + col, w, left, p.wide);
#pragma unroll
        for (int j = 0; j < 8; ++j) out[2 * j] = bf16_lo(w[j]), out[2 * j + 1] = bf16_hi(w[j]);
      }
      // (all of them asked for before the first is used)
      float4 f[S][4];
#pragma unroll
      for (int q = 0; q < S; ++q) {
        const uint32_t from = ptx::map_to_rank(ptx::smem_u32(part + ((c / 4) * kBM + row) * 4), q);
#pragma unroll
        for (int j = 0; j < 4; ++j) f[q][j] = ld_cluster(from + j * kBM * 16);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
#pragma unroll
        for (int q = 1; q < S; ++q) f[0][j].x += f[q][j].x, f[0][j].y += f[q][j].y, f[0][j].z += f[q][j].z, f[0][j].w += f[q][j].w;
        v[4 * j] = f[0][j].x, v[4 * j + 1] = f[0][j].y, v[4 * j + 2] = f[0][j].z, v[4 * j + 3] = f[0][j].w;
      }
      if (left <= 0) continue;
      if (p.bias != nullptr) {
        float b[8];
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          if (left <= g * 8) break;
          Vec<__nv_bfloat16>::unpack(*reinterpret_cast<const uint4*>(p.bias + col + g * 8), b);
#pragma unroll
          for (int j = 0; j < 8; ++j) v[g * 8 + j] += b[j];
        }
      }
      if (p.z != nullptr) {
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = pack_bf16x2(v[2 * j], v[2 * j + 1]);
        write16(p.z + grow * p.pz + col, w, left, p.wide);
      }
#pragma unroll
      for (int j = 0; j < 16; j += 2) act2<ACT, false>(v[j], v[j + 1]);
      if constexpr (DROP) {
        const uint64_t g0 = static_cast<uint64_t>(p.first + grow * p.step + col) >> 3, group[2] = {g0, g0 + 1};
        philox<2>(stream, group, w);
#pragma unroll
        for (int j = 0; j < 8; ++j) add_kept2(out[2 * j], out[2 * j + 1], v[2 * j], v[2 * j + 1], w[j], p.drop);
      } else {
#pragma unroll
        for (int j = 0; j < 16; ++j) out[j] += v[j];
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) w[j] = pack_bf16x2(out[2 * j], out[2 * j + 1]);
      write16(p.y + grow * p.py + col, w, left, p.wide);
    }
  }
  ptx::cluster_sync_all();   // no CTA leaves while another may still read its sums
}

// How a product is cut.
struct Plan {
  bool pair;
  int BN, split;   // split > 1: K shared among so many CTAs
};

// Cycles of an SM for the epilogue of 128 tokens by bn channels.
double epilogue_cycles(const LinearCall& c, int bn) {
  return bn * (10.0 + (c.act != LBP_ACT_NONE ? 16.0 : 0.0) + (c.drop.on ? 12.0 : 0.0)) + 500.0;
}

Plan choose_plan(const LinearCall& c, int sms) {
  const int num_kb = (c.Cin + kBK - 1) / kBK;
  Plan best{false, 64, 1};
  double least = -1.0;
  for (int pair = 0; pair < 2; ++pair) {
    if (pair && (c.rows <= kBM || sms < 2)) continue;
    const int bm = pair ? 2 * kBM : kBM, units = pair ? sms / 2 : sms;
    for (int bn = 64; bn <= 256; bn += 64) {
      if (bn > 64 && bn - 64 >= c.Cout) continue;   // wider than the matrix
      const long long tiles = ((c.rows + bm - 1) / bm) * ((c.Cout + bn - 1) / bn);
      const double rounds = static_cast<double>((tiles + units - 1) / units);
      // cycles of an SM: a k-block's products and operands (60 bytes a cycle), an element's epilogue
      const double mma = 2.0 * bn, load = (kABytes + (pair ? bn / 2 : bn) * kBK * 2) / 60.0;
      const double main = num_kb * (mma > load ? mma : load) + 200.0;
      const double epi = epilogue_cycles(c, bn);
      const double cost = rounds * (main > epi ? main : epi) + (main > epi ? epi : main) + 1500.0;
      if (least < 0.0 || cost < least) {
        least = cost;
        best = Plan{pair != 0, bn, 1};
      }
    }
  }
  // K shared: one round, for the price of the exchange (fitted to 3072 -> 768 and 768 -> 768 channels at 33 to 1024
  // tokens, us unshared / shared: 11.2 / 6.3 and 5.5 / 4.5 at 64, 11.7 / 8.2 and 6.0 / 6.5 at 300, 12.4 / 10.4 at 1024; 768 -> 3072
  // at 64: 5.6 / 7.0).  Clusters that are resident at once, at a CTA to an SM: 74 of two and 33 of four on the GPU at
  // hand; others have GPCs of other sizes.
  constexpr int kClusters[5] = {0, 0, 72, 0, 30};
  for (int bn = 64; bn <= 128; bn += 64) {
    if (bn > 64 && c.Cout <= 64) continue;
    const long long tiles = ((c.rows + kBM - 1) / kBM) * ((c.Cout + bn - 1) / bn);
    for (int S = 2; S <= 4; S *= 2) {
      if (tiles > kClusters[S] || S > num_kb) continue;
      const double cost = (num_kb + S - 1) / S * ((kABytes + bn * kBK * 2) / 60.0) + (S == 2 ? 7000.0 : bn == 64 ? 4600.0 : 8000.0);
      if (cost < least) {
        least = cost;
        best = Plan{false, bn, S};
      }
    }
  }
  return best;
}

}  // namespace

static thread_local int g_test_stall = 0;

int launch_linear_umma(const LinearCall& c, cudaStream_t stream) {
  int dev = 0, sms = 0;
  LBP_CUDA_TRY(cudaGetDevice(&dev));
  LBP_CUDA_TRY(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
  const Plan plan = choose_plan(c, sms);
  const int ctas = plan.pair ? 2 : 1, part = plan.BN / ctas;
  Params p{};
  p.bias = static_cast<const __nv_bfloat16*>(c.bias);
  p.rows = c.rows;
  p.Cout = c.Cout;
  p.BN = plan.BN;
  p.num_kb = (c.Cin + kBK - 1) / kBK;
  p.tiles_n = (c.Cout + plan.BN - 1) / plan.BN;
  const long long tiles = ((c.rows + ctas * kBM - 1) / (ctas * kBM)) * p.tiles_n;
  if (tiles >= (1ll << 31)) return LBP_ERR_SHAPE;
  p.tiles = static_cast<int32_t>(tiles);
  p.stage_bytes = kABytes + part * kBK * 2;
  const int room = kSmemMax - kBarBytes - kBiasBytes - kOutBytes;
  p.stages = room / p.stage_bytes < kMaxStages ? room / p.stage_bytes : kMaxStages;
  p.test_stall = g_test_stall;
  p.first = c.first;
  p.step = c.step;
  p.drop = c.drop;
  p.status = c.status;
  p.residual = static_cast<const __nv_bfloat16*>(c.residual);
  p.y = static_cast<__nv_bfloat16*>(c.y);
  p.z = static_cast<__nv_bfloat16*>(c.z);
  p.pr = c.pr;
  p.py = c.py;
  p.pz = c.pz;
  auto wide = [](const void* q, int64_t pitch) { return ((reinterpret_cast<uintptr_t>(q) | static_cast<uintptr_t>(2 * pitch)) & 31u) == 0; };
  p.wide = c.residual == nullptr || wide(c.residual, c.pr);
  if (plan.split > 1) p.wide = p.wide && wide(c.y, c.py) && (c.z == nullptr || wide(c.z, c.pz));
  Maps tm;
  if (int e = encode_matrix_tensor_map(&tm.x, c.x, c.rows, c.Cin, kBM, c.px)) return e;
  if (int e = encode_matrix_tensor_map(&tm.W, c.W, c.Cout, c.Cin, part)) return e;
  tm.y = tm.z = tm.x;
  if (plan.split == 1)   // (else by plain stores)
    if (int e = encode_matrix_tensor_map(&tm.y, c.y, c.rows, c.Cout, 32, c.py, c.z != nullptr ? 32 : 64)) return e;
  if (plan.split == 1 && c.z != nullptr)
    if (int e = encode_matrix_tensor_map(&tm.z, c.z, c.rows, c.Cout, 32, c.pz, 32)) return e;

  const int units = plan.pair ? sms / 2 : sms;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = plan.split > 1 ? plan.split : 2;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.gridDim = dim3(static_cast<unsigned>(ctas * (tiles < units ? tiles : units)));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = p.stages * p.stage_bytes + kBiasBytes + kOutBytes + kBarBytes;
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = plan.pair || plan.split > 1 ? 2 : 1;
  if (plan.split > 1) {
    cfg.gridDim = dim3(static_cast<unsigned>(tiles) * plan.split);
    cfg.blockDim = dim3(kSplitThreads);
    cfg.dynamicSmemBytes = kSplitSmem;
  }
  return with_act(c.act, [&](auto a) -> int {
    constexpr int ACT = decltype(a)::value;
    auto launch = [&](auto kern, PerDevice& configured) -> int {
      if (int e = allow_dynamic_smem(configured, reinterpret_cast<const void*>(kern), kSmemMax)) return e;
      LBP_CUDA_TRY(cudaLaunchKernelEx(&cfg, kern, tm, p));
      count_launch();
      return LBP_OK;
    };
    if (plan.split > 1) {
      static PerDevice split_configured[4];
      if (plan.split == 2)
        return c.drop.on ? launch(linear_split_kernel<ACT, true, 2>, split_configured[1])
                         : launch(linear_split_kernel<ACT, false, 2>, split_configured[0]);
      return c.drop.on ? launch(linear_split_kernel<ACT, true, 4>, split_configured[3])
                       : launch(linear_split_kernel<ACT, false, 4>, split_configured[2]);
    }
    static PerDevice configured[16];
    auto by = [&](auto drop, auto res, auto zy) -> int {
      constexpr bool DROP = decltype(drop)::value, RES = decltype(res)::value, ZY = decltype(zy)::value;
      PerDevice* const d = configured + 2 * (4 * DROP + 2 * RES + ZY);
      return plan.pair ? launch(linear_umma_kernel<ACT, DROP, RES, ZY, true>, d[1])
                       : launch(linear_umma_kernel<ACT, DROP, RES, ZY, false>, d[0]);
    };
    auto by_z = [&](auto drop, auto res) -> int {
      return c.z != nullptr ? by(drop, res, std::true_type{}) : by(drop, res, std::false_type{});
    };
    if (c.drop.on)
      return c.residual != nullptr ? by_z(std::true_type{}, std::true_type{}) : by_z(std::true_type{}, std::false_type{});
    return c.residual != nullptr ? by_z(std::false_type{}, std::true_type{}) : by_z(std::false_type{}, std::false_type{});
  });
}

}  // namespace layer

void set_test_stall_linear(int mode) { layer::g_test_stall = mode; }

}  // namespace lbp
