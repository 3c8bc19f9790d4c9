// 8-bit (and fp16, bf16) matrix products of many rows.  Bound by the tensor cores.
// A cluster of two CTAs owns tiles of 256 output features x up to 256 rows (tcgen05.mma.cta_group::2): CTA r holds features 128 r ..
// of the tile (A operand and accumulators) and loads half of its rows (B operand), which both read.  The instruction takes as many
// rows as the tile has, in multiples of 32, and lists are cut into tiles of even size.  The grid is persistent;
// tiles of one expert follow each other with its row tiles first, so that the CTAs that run at once share its weights.
// Which tiles there are is worked out by every cluster from the experts' offsets, which the host does not know.
// Roles per CTA: warp 0 loads, warp 1 (of CTA 0) multiplies, warp 2 allocates tensor memory, warp 3 plans, warps 4-11 write y:
// warp w the features of quarter w % 4, every other 32 rows; warps 12-15, where a list says which rows of x, bring those.
// Accumulators alternate, so that writing one overlaps the next.
// A ring slot holds kSub blocks of 128 bytes of K: one round of barriers per 8 instructions (with a block per slot and six slots
// 8192 x 4096 x 4096 takes 97 us, so 89).  The instruction takes as long for few rows as for 256 (a block of K 0.28 us with 32 rows, 0.40
// with 256, at which point 32 KB per SM and block come out of L2 at 11 TB/s): few full tiles beat many small ones.
// Waits are bounded; a tile whose wait runs out is written as NaN.
#include "matmul_common.cuh"

namespace bl {

namespace {

using namespace mm;

constexpr int kThreads = 384, kGatherWarps = 4;       // the latter only where a list says which rows of x
constexpr int kPairFeatures = 256;
constexpr int kHalf = 128;                           // features per CTA
constexpr int kSub = 2;
constexpr int kABytes = kHalf * kRowBytes;
constexpr int kEpiWarps = 8;

constexpr int kMostRows = 256, kUnit = 32;             // of a tile: most, and what its size is a multiple of
constexpr int kBBytes = kMostRows / 2 * kRowBytes;
constexpr int kStage = kABytes + kBBytes;
constexpr int kSlotBytes = kSub * kStage;
constexpr int kSlots = 3;

__device__ __forceinline__ int padded(int rows) { return (rows + kUnit - 1) / kUnit * kUnit; }

struct Control {
  unsigned long long full[kSlots], empty[kSlots];               // full: rank 0's, for the bytes of both
  unsigned long long gathered[kSlots];                          // this CTA's rows by a list
  unsigned long long tmem_full[2], tmem_empty[2], drained;      // tmem_empty: rank 0's, for the warps of both
  uint32_t tmem_base;
  int abort_flag;
  uint32_t filled, relayed;                                     // slots that warp 0, and with listed rows warp 3, reported to full
  alignas(16) float x_scale[kEpiWarps][32];
};
inline size_t smem_bytes(int experts) { return 1024 + (size_t)kSlots * kSlotBytes + sizeof(Control) + plan_bytes(experts); }

template <bool kInt, typename TY>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads + 32 * kGatherWarps, 1)
matmul_wide_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x, MatmulArgs a, uint32_t idesc,
                   int feature_tiles, int tile_rows, int tx_bytes, long long polls) {
  constexpr int kTmemCols = 2 * kMostRows;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  Control* ctl = reinterpret_cast<Control*>(smem + (size_t)kSlots * kSlotBytes);
  int* plan = reinterpret_cast<int*>(ctl + 1);
  volatile int* abort_flag = &ctl->abort_flag;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_rank();
  if (threadIdx.x == 0) {
    prefetch_map(&map_w);
    prefetch_map(&map_x);
    for (int s = 0; s < kSlots; ++s) {
      mbar_init(smem_u32(&ctl->full[s]), a.rows ? 4 : 2);
      mbar_init(smem_u32(&ctl->empty[s]), 1);
      mbar_init(smem_u32(&ctl->gathered[s]), 32 * kGatherWarps);
    }
    for (int b = 0; b < 2; ++b) { mbar_init(smem_u32(&ctl->tmem_full[b]), 1); mbar_init(smem_u32(&ctl->tmem_empty[b]), 2 * kEpiWarps); }
    mbar_init(smem_u32(&ctl->drained), 1);
    ctl->abort_flag = polls == 0;
    ctl->filled = ctl->relayed = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 2) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ctl->tmem_base)), "r"(kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    pdl_launch_dependents();                       // not before the tensor memory is ours: a kernel behind this one may take some, then wait for this one
  }
  if (warp == 3 && !a.offsets) make_plan(a, plan, tile_rows);
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();                                // both CTAs' barriers exist before any remote arrival
  tc_fence_after();
  // So far nothing that the kernel before this one on the stream could have written was read.
  pdl_wait();
  if (a.offsets) {
    if (warp == 3) make_plan(a, plan, tile_rows);
    __syncthreads();
  }
  const uint32_t tmem_base = ctl->tmem_base;
  // Bounded; who gives up lets both CTAs know.
  const uint32_t partner_flag = map_to_rank(smem_u32(&ctl->abort_flag), rank ^ 1u);
  auto wait = [&](uint32_t bar, uint32_t parity) {
    if (mbar_wait_polls(bar, parity, abort_flag, polls)) return true;
    st_cluster(partner_flag, 1u);
    return false;
  };
  const int blocks = (int)((a.K * (kInt ? 1 : 2) + kRowBytes - 1) / kRowBytes);

  if (polls == 0 && (warp < 4 || warp >= 4 + kEpiWarps)) {
    // no waits allowed: nothing is started
  } else if (warp == 0) {
    if (lane == 0) {
      int slot = 0;
      uint32_t phase = 0, filled = 0;
      const uint32_t full0 = map_to_rank(smem_u32(&ctl->full[0]), 0);
      bool ok = true;
      for (Walk w(plan, a.experts, feature_tiles, blockIdx.x >> 1, gridDim.x >> 1); ok && w.valid(); w.next()) {
        w.locate(kUnit);
        const int n0 = w.f * kPairFeatures + (int)rank * kHalf, mine = (int)rank * (padded(w.rows) / 2);     // this CTA's features and rows of the tile
        for (int kb = 0; kb < blocks; kb += kSub) {
          const int n = min(kSub, blocks - kb);
          const uint32_t bar = full0 + 8u * (uint32_t)slot;
          ok = wait(smem_u32(&ctl->empty[slot]), phase ^ 1u);
          if (!ok) break;
          mbar_arrive_expect_tx_cluster(bar, (uint32_t)(tx_bytes * n));
          for (int b = 0; b < n; ++b) {
            const uint32_t dst = smem_u32(smem + (size_t)slot * kSlotBytes + (size_t)b * kStage);
            const int c = (kb + b) * kRowBytes;
            tma_load_4d_pair(dst, &map_w, c, n0, 0, w.e, bar);
            if (!a.rows) tma_load_2d_pair(dst + kABytes, &map_x, c, w.row0 + mine, bar);
          }
          ++filled;
          if (++slot == kSlots) { slot = 0; phase ^= 1u; }
        }
      }
      ctl->filled = filled;
      // The last products report their slots to both CTAs: this one is there until they have.
      for (uint32_t i = filled > kSlots ? filled - kSlots : 0u; ok && i < filled; ++i) ok = wait(smem_u32(&ctl->empty[i % kSlots]), i / kSlots & 1u);
    }
    __syncwarp();
  } else if (warp == 1) {
    if (lane == 0 && rank == 0) {
      int slot = 0;
      uint32_t phase = 0, pass = 0;
      bool ok = true;
      const uint32_t empty0 = map_to_rank(smem_u32(&ctl->empty[0]), 0), empty1 = map_to_rank(smem_u32(&ctl->empty[0]), 1);
      const uint32_t done0 = map_to_rank(smem_u32(&ctl->tmem_full[0]), 0), done1 = map_to_rank(smem_u32(&ctl->tmem_full[0]), 1);
      for (Walk w(plan, a.experts, feature_tiles, blockIdx.x >> 1, gridDim.x >> 1); ok && w.valid(); w.next(), ++pass) {
        const uint32_t buf = pass & 1u, d = tmem_base + buf * (uint32_t)kMostRows;
        w.locate(kUnit);
        const uint32_t desc = idesc | (uint32_t)(padded(w.rows) >> 3) << 17;
        if (!(ok = wait(smem_u32(&ctl->tmem_empty[buf]), ((pass >> 1) & 1u) ^ 1u))) break;
        tc_fence_after();
        for (int kb = 0; kb < blocks; kb += kSub) {
          if (!(ok = wait(smem_u32(&ctl->full[slot]), phase))) break;
          tc_fence_after();
          const uint32_t at = smem_u32(smem + (size_t)slot * kSlotBytes);
          const int n = min(kSub, blocks - kb);
          for (int b = 0; b < n; ++b) {
            const uint64_t adesc = smem_desc_sw128(at + (uint32_t)(b * kStage)), bdesc = smem_desc_sw128(at + (uint32_t)(b * kStage + kABytes));
#pragma unroll
            for (int j = 0; j < kRowBytes / 32; ++j)
              mma<kInt, 2>(d, adesc + (uint64_t)(2 * j), bdesc + (uint64_t)(2 * j), desc, kb > 0 || b > 0 || j > 0);
          }
          mma_commit_pair(empty0 + 8u * (uint32_t)slot);
          mma_commit_pair(empty1 + 8u * (uint32_t)slot);
          if (++slot == kSlots) { slot = 0; phase ^= 1u; }
        }
        if (!ok) break;
        mma_commit_pair(done0 + 8u * buf);
        mma_commit_pair(done1 + 8u * buf);
      }
      // The products are over before the memory that they use is given back, whoever gave up waiting for them.
      mma_commit_pair(map_to_rank(smem_u32(&ctl->drained), 0));
      mbar_wait_quiet(smem_u32(&ctl->drained), 0);
    }
    __syncwarp();
  } else if (warp >= 4 + kEpiWarps) {
    // Rows by a list: 16-byte copies, eight lanes to a row of 128 bytes (a tensor copy of four listed rows takes 65 clocks, three
    // times what the tensor cores leave: 8192 rows x 2048 x 8192, 512 for each of 16 experts, 316 us, with these copies 127).
    constexpr int kPer = kMostRows / 2 * 8 / (32 * kGatherWarps);  // copies per thread and block of K, at most
    const int u = threadIdx.x - 32 * (4 + kEpiWarps), part = u & 7;
    const int64_t row_bytes = a.K * (kInt ? 1 : 2);
    const char* x = reinterpret_cast<const char*>(a.x);
    int slot = 0;
    uint32_t phase = 0;
    bool ok = true;
    for (Walk w(plan, a.experts, feature_tiles, blockIdx.x >> 1, gridDim.x >> 1); ok && w.valid(); w.next()) {
      w.locate(kUnit);
      const int passes = padded(w.rows) / kUnit;       // of 16 rows of this CTA's half
      const char* from[kPer];
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int row = (int)rank * (padded(w.rows) / 2) + i * 4 * kGatherWarps + (u >> 3);
        from[i] = x + (int64_t)source_row(a, w.row0 + min(row, w.rows - 1)) * a.ld_x * (kInt ? 1 : 2) + part * 16;
      }
      for (int kb = 0; kb < blocks; kb += kSub) {
        const int n = min(kSub, blocks - kb);
        if (lane == 0) ok = wait(smem_u32(&ctl->empty[slot]), phase ^ 1u);
        ok = __shfl_sync(0xFFFFFFFFu, ok, 0);
        if (!ok) break;
        for (int b = 0; b < n; ++b) {
          const uint32_t dst = smem_u32(smem + (size_t)slot * kSlotBytes + (size_t)b * kStage + kABytes);
          const int64_t at = (int64_t)(kb + b) * kRowBytes;
          const uint32_t bytes = at + part * 16 < row_bytes ? 16u : 0u;       // behind the row: zeros
          const int64_t skip = bytes ? at : 0;
#pragma unroll
          for (int i = 0; i < kPer; ++i) {
            if (i >= passes) break;
            const int row = i * 4 * kGatherWarps + (u >> 3);
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst + (uint32_t)(row * kRowBytes + ((part ^ (row & 7)) << 4))),
                         "l"(from[i] + skip), "r"(bytes) : "memory");
          }
        }
        asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(&ctl->gathered[slot])) : "memory");
        if (++slot == kSlots) { slot = 0; phase ^= 1u; }
      }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
  } else if (warp == 3) {
    // Rows by a list: hands the copies of a slot over to the tensor cores' side of memory and reports them.
    if (lane == 0 && a.rows) {
      int slot = 0;
      uint32_t phase = 0, relayed = 0;
      bool ok = true;
      const uint32_t full0 = map_to_rank(smem_u32(&ctl->full[0]), 0);
      for (Walk w(plan, a.experts, feature_tiles, blockIdx.x >> 1, gridDim.x >> 1); ok && w.valid(); w.next()) {
        for (int kb = 0; kb < blocks; kb += kSub) {
          if (!(ok = wait(smem_u32(&ctl->gathered[slot]), phase))) break;
          fence_proxy_async_smem();
          mbar_arrive_cluster(full0 + 8u * (uint32_t)slot);
          ++relayed;
          if (++slot == kSlots) { slot = 0; phase ^= 1u; }
        }
      }
      ctl->relayed = relayed;
    }
    __syncwarp();
  } else if (warp >= 4) {
    const int quarter = warp & 3, half = (warp - 4) >> 2;
    const int f = quarter * 32 + lane, c0 = half * 32;      // feature of this CTA, first row of the tile
    float* x_scale = ctl->x_scale[warp - 4];
    TY* y = reinterpret_cast<TY*>(a.y);
    const TY* res = reinterpret_cast<const TY*>(a.residual);
    bool ok = polls != 0;
    uint32_t pass = 0;
    const uint32_t release = map_to_rank(smem_u32(&ctl->tmem_empty[0]), 0);
    for (Walk w(plan, a.experts, feature_tiles, blockIdx.x >> 1, gridDim.x >> 1); w.valid(); w.next(), ++pass) {
      w.locate(kUnit);
      const uint32_t buf = pass & 1u;
      const int n = w.f * kPairFeatures + (int)rank * kHalf + f;
      const Feature<TY> feature(a, w.e, n);
      float scale_of[kMostRows / 64];                  // of row c0 + 64 i + lane
      if (kInt) {
#pragma unroll
        for (int i = 0; i < kMostRows / 64; ++i)
          scale_of[i] = a.x_scale && c0 + 64 * i + lane < w.rows ? a.x_scale[source_row(a, w.row0 + c0 + 64 * i + lane)] : 1.f;
      }
      if (ok) {
        if (lane == 0) ok = wait(smem_u32(&ctl->tmem_full[buf]), (pass >> 1) & 1u);
        ok = __shfl_sync(0xFFFFFFFFu, ok, 0);
      }
      tc_fence_after();
      const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16) + buf * (uint32_t)kMostRows;
#pragma unroll 1
      for (int i = 0; c0 + 64 * i < w.rows; ++i) {
        const int c = c0 + 64 * i;
        // A chunk of 32 rows without a branch in between: its loads and its conversions overlap.
        const int here = w.rows - c;                   // rows of the chunk that exist, if under 32
        const int64_t row = w.row0 + c;
        Raw<TY> add[32];
        if (res && feature.on) {
          const TY* from = res + row * a.ld_res + n;
          if (here >= 32) {
#pragma unroll
            for (int j = 0; j < 32; ++j) add[j] = load_raw(from + j * a.ld_res);
          } else {
#pragma unroll
            for (int j = 0; j < 32; ++j) add[j] = load_raw(from + min(j, here - 1) * a.ld_res);
          }
        }
        uint32_t r[32];
        tmem_ld32(taddr + (uint32_t)c, r);
        if (kInt) {
          __syncwarp();
          x_scale[lane] = i == 0 ? scale_of[0] : i == 1 ? scale_of[1] : i == 2 ? scale_of[2] : scale_of[3];
          __syncwarp();
        }
        float v[32];
#pragma unroll
        for (int j = 0; j < 32; j += 4) {
          const float4 s = kInt ? *reinterpret_cast<const float4*>(x_scale + j) : make_float4(1.f, 1.f, 1.f, 1.f);
          feature.finish2(sum_value<kInt>(r[j]), sum_value<kInt>(r[j + 1]), s.x, s.y, v[j], v[j + 1]);
          feature.finish2(sum_value<kInt>(r[j + 2]), sum_value<kInt>(r[j + 3]), s.z, s.w, v[j + 2], v[j + 3]);
        }
        if (res) {
#pragma unroll
          for (int j = 0; j < 32; ++j) v[j] += raw_value<TY>(add[j]);
        }
        if (!ok) {
#pragma unroll
          for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(0x7FC00000u);
        }
        TY* out = y + row * a.ld_y + n;
        if (feature.on && here >= 32) {
#pragma unroll
          for (int j = 0; j < 32; ++j) out[j * a.ld_y] = out_cast<TY>(v[j]);
        } else if (feature.on) {
#pragma unroll
          for (int j = 0; j < 32; ++j)
            if (j < here) out[j * a.ld_y] = out_cast<TY>(v[j]);
        }
      }
      // One that gave up reports nothing more: its report would stand for a warp, of either CTA, that still reads, and the next products
      // would go over what that one reads.  The multiplying warp gives up as well then, and every tile from here on is NaN.
      tc_fence_before();
      __syncwarp();
      if (ok && lane == 0) mbar_arrive_cluster(release + 8u * buf);
    }
  }

  tc_fence_before();
  __syncthreads();
  cluster_sync_all();                                // the partner no longer touches this CTA's memory
  if (*abort_flag && polls != 0) {
    // A wait ran out, whichever role's and however late, and both CTAs know it: copies may be on their way that no product waited for.
    // They are counted on rank 0's barriers, whose phases still lack the reports that nobody made: rank 0 makes those, then waits.  Only
    // the last round of the ring can be open: a slot is filled again when the products have read it.
    if (rank == 0 && threadIdx.x == 0) {
      const uint32_t reports[4] = {ctl->filled, ld_cluster(map_to_rank(smem_u32(&ctl->filled), 1)), ctl->relayed,
                                   ld_cluster(map_to_rank(smem_u32(&ctl->relayed), 1))};
      const uint32_t most = max(max(reports[0], reports[1]), max(reports[2], reports[3]));
      for (uint32_t i = most > kSlots ? most - kSlots : 0u; i < most; ++i) {
        const uint32_t bar = smem_u32(&ctl->full[i % kSlots]);
        for (int r = 0; r < (a.rows ? 4 : 2); ++r)
          if (reports[r] <= i) mbar_arrive(bar);
        mbar_wait_quiet(bar, i / kSlots & 1u);
      }
    }
    cluster_sync_all();
  }
  if (warp == 2) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(kTmemCols) : "memory");
  }
}

template <bool kInt, typename TY>
cudaError_t launch(const MatmulArgs& a, int tile_rows, cudaStream_t s) {
  const int es = kInt ? 1 : 2;
  const int64_t feature_tiles = (a.N + kPairFeatures - 1) / kPairFeatures;
  int64_t token_tiles = (a.R + tile_rows - 1) / tile_rows;
  if (a.offsets) token_tiles = a.R / tile_rows + (a.experts < a.R ? a.experts : a.R);    // at most: one that is not full per expert
  const int64_t tiles = token_tiles * feature_tiles;
  if (tiles > 0x7FFFFFFF) return cudaErrorInvalidValue;
  CUtensorMap map_w, map_x;
  const int box_n = a.N < kHalf ? (int)a.N : kHalf, box_t = a.x_rows < tile_rows / 2 ? (int)a.x_rows : tile_rows / 2;
  cudaError_t e = encode_blocks(&map_w, a.w, a.K * es, a.N, a.ld_w * es, a.experts, a.expert_stride * es, box_n, 0);
  if (e == cudaSuccess) e = encode_rows(&map_x, a.x, a.K * es, a.x_rows, a.ld_x * es, box_t);
  if (e != cudaSuccess) return e;
  const int tx = (box_n + (a.rows ? 0 : box_t)) * kRowBytes;
  const unsigned threads = kThreads + (a.rows ? 32 * kGatherWarps : 0);
  const auto kern = matmul_wide_kernel<kInt, TY>;
  // Clusters that the device holds at once; 0 until the kernel is set up there.  Devices beyond the table are set up on every call.
  static std::atomic<int> resident[64];
  int dev = 0;
  if ((e = cudaGetDevice(&dev)) != cudaSuccess) return e;
  int cap = dev < 64 ? resident[dev].load(std::memory_order_acquire) : 0;
  if (cap == 0) {
    const size_t most = smem_bytes(kMaxExperts);
    if ((e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most)) != cudaSuccess) return e;
    if ((e = max_clusters(kern, 2, kThreads + 32 * kGatherWarps, most, &cap)) != cudaSuccess) return e;
    if (cap < 1) return cudaErrorInvalidConfiguration;
    if (dev < 64) resident[dev].store(cap, std::memory_order_release);
  }
  const int64_t clusters = tiles < cap ? tiles : cap;
  const long long polls = g_debug_wait_polls.load(std::memory_order_relaxed);
  return launch_pdl(kern, dim3((unsigned)(2 * clusters)), threads, smem_bytes(a.experts), s, map_w, map_x, a,
                    instr_desc(a.operand, kPairFeatures, 0), (int)feature_tiles, tile_rows, tx, polls);
}

}  // namespace

cudaError_t launch_matmul_wide(const MatmulArgs& a, int tile_rows, cudaStream_t s) {
  const bool whole = a.operand == BL_I8;
  switch (a.yt) {
    case BL_F32: return whole ? launch<true, float>(a, tile_rows, s) : launch<false, float>(a, tile_rows, s);
    case BL_F16: return whole ? launch<true, __half>(a, tile_rows, s) : launch<false, __half>(a, tile_rows, s);
    default: return whole ? launch<true, __nv_bfloat16>(a, tile_rows, s) : launch<false, __nv_bfloat16>(a, tile_rows, s);
  }
}

}  // namespace bl
