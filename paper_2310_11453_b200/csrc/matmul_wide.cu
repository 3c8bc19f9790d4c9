// 8-bit (and fp16, bf16) matrix products of many rows.  Bound by the tensor cores.
// A cluster of two CTAs owns tiles of 256 output features x kTokens rows (tcgen05.mma.cta_group::2): CTA r holds features 128 r ..
// of the tile (A operand and accumulators) and loads half of its rows (B operand), which both read.  The grid is persistent;
// tiles of one expert follow each other with its row tiles first, so that the CTAs that run at once share its weights.
// Which tiles there are is worked out by every cluster from the experts' offsets, which the host does not know.
// Roles per CTA: warp 0 loads, warp 1 (of CTA 0) multiplies, warp 2 allocates tensor memory, warp 3 plans, warps 4-11 write y:
// warp w the features of quarter w % 4 and half of the rows; warps 12-15, where a list says which rows of x, bring those.  Accumulators alternate, so that writing one overlaps the next.
// A ring slot holds kSub blocks of 128 bytes of K: one round of barriers per 8 instructions.
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
constexpr int kMaxSlots = 4;

template <int kTokens> constexpr int kBBytes = kTokens / 2 * kRowBytes;
template <int kTokens> constexpr int kSlotBytes = kSub * (kABytes + kBBytes<kTokens>);
template <int kTokens> constexpr int kSlots = 196608 / kSlotBytes<kTokens>;

struct Control {
  unsigned long long full[kMaxSlots], empty[kMaxSlots];          // full: rank 0's, for the bytes of both
  unsigned long long gathered[kMaxSlots];                        // this CTA's rows by a list
  unsigned long long tmem_full[2], tmem_empty[2], drained;       // tmem_empty: rank 0's, for the warps of both
  uint32_t tmem_base;
  int abort_flag;
  alignas(16) float x_scale[kEpiWarps][128];
};
// Per expert the first tile, the first row and the number of rows.
inline size_t plan_bytes(int experts) { return (size_t)(3 * experts + 1) * sizeof(int); }
template <int kTokens>
inline size_t smem_bytes(int experts) { return 1024 + (size_t)kSlots<kTokens> * kSlotBytes<kTokens> + sizeof(Control) + plan_bytes(experts); }

struct Walk {                                        // this cluster's tiles, in the order in which every role of both CTAs takes them
  const int *first, *start, *count;
  uint32_t t, total, stride, feature_tiles;
  int e, row0, rows, f;
  __device__ Walk(const int* plan, int experts, uint32_t feature_tiles_)
      : first(plan), start(plan + experts + 1), count(plan + 2 * experts + 1), t(blockIdx.x >> 1),
        total((uint32_t)plan[experts] * feature_tiles_), stride(gridDim.x >> 1), feature_tiles(feature_tiles_), e(0), row0(0), rows(0), f(0) {}
  __device__ bool valid() const { return t < total; }
  __device__ void next() { t += stride; }
  __device__ void locate(int tile_rows) {
    while (t >= feature_tiles * (uint32_t)first[e + 1]) ++e;
    const uint32_t local = t - feature_tiles * (uint32_t)first[e], n = (uint32_t)(first[e + 1] - first[e]);
    f = (int)(local / n);
    const int skip = (int)(local - (uint32_t)f * n) * tile_rows;
    row0 = start[e] + skip;
    rows = min(tile_rows, count[e] - skip);
  }
};

template <int kTokens, bool kInt, typename TY>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads + 32 * kGatherWarps, 1)
matmul_wide_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x, MatmulArgs a, uint32_t idesc,
                   int feature_tiles, int tx_bytes, long long polls) {
  constexpr int kHalfRows = kTokens / 2;
  constexpr int kStage = kABytes + kBBytes<kTokens>;
  constexpr int kNSlots = kSlots<kTokens>;
  constexpr int kTmemCols = 2 * kTokens;
  static_assert(kNSlots <= kMaxSlots, "barriers");
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  Control* ctl = reinterpret_cast<Control*>(smem + (size_t)kNSlots * kSlotBytes<kTokens>);
  int* plan = reinterpret_cast<int*>(ctl + 1);
  volatile int* abort_flag = &ctl->abort_flag;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_rank();
  pdl_launch_dependents();
  if (threadIdx.x == 0) {
    prefetch_map(&map_w);
    prefetch_map(&map_x);
    for (int s = 0; s < kNSlots; ++s) {
      mbar_init(smem_u32(&ctl->full[s]), a.rows ? 4 : 2);
      mbar_init(smem_u32(&ctl->empty[s]), 1);
      mbar_init(smem_u32(&ctl->gathered[s]), 32 * kGatherWarps);
    }
    for (int b = 0; b < 2; ++b) { mbar_init(smem_u32(&ctl->tmem_full[b]), 1); mbar_init(smem_u32(&ctl->tmem_empty[b]), 2 * kEpiWarps); }
    mbar_init(smem_u32(&ctl->drained), 1);
    ctl->abort_flag = polls == 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 2) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ctl->tmem_base)), "r"(kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  pdl_wait();
  if (warp == 3) {
    int *first = plan, *start = plan + a.experts + 1, *count = plan + 2 * a.experts + 1;
    int seen = 0;
    for (int base = 0; base < a.experts; base += 32) {
      const int e = base + lane;
      int from = 0, n = 0;
      if (e < a.experts) {
        if (a.offsets) {
          from = offset_of(a.offsets, e, (int)a.R);
          n = max(0, offset_of(a.offsets, e + 1, (int)a.R) - from);
        } else {
          n = (int)a.R;
        }
        start[e] = from;
        count[e] = n;
      }
      const int tiles = (n + kTokens - 1) / kTokens;
      int upto = tiles;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xFFFFFFFFu, upto, o);
        if (lane >= o) upto += v;
      }
      if (e < a.experts) first[e] = seen + upto - tiles;
      seen += __shfl_sync(0xFFFFFFFFu, upto, 31);
    }
    if (lane == 0) first[a.experts] = seen;
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();                                // both CTAs' barriers exist before any remote arrival
  tc_fence_after();
  const uint32_t tmem_base = ctl->tmem_base;
  const int blocks = (int)((a.K * (kInt ? 1 : 2) + kRowBytes - 1) / kRowBytes);

  if (*abort_flag && (warp < 4 || warp >= 4 + kEpiWarps)) {
    // no waits allowed: nothing is started
  } else if (warp == 0) {
    if (lane == 0) {
    int slot = 0;
    uint32_t phase = 0;
    const uint32_t full0 = map_to_rank(smem_u32(&ctl->full[0]), 0);
    bool ok = true;
    for (Walk w(plan, a.experts, (uint32_t)feature_tiles); ok && w.valid(); w.next()) {
      w.locate(kTokens);
      const int n0 = w.f * kPairFeatures + (int)rank * kHalf, mine = (int)rank * kHalfRows;     // this CTA's features and rows of the tile
      for (int kb = 0; kb < blocks; kb += kSub) {
        const int n = min(kSub, blocks - kb);
        const uint32_t bar = full0 + 8u * (uint32_t)slot;
        ok = wait_for(smem_u32(&ctl->empty[slot]), phase ^ 1u, abort_flag, polls);
        if (!ok) break;
        mbar_arrive_expect_tx_cluster(bar, (uint32_t)(tx_bytes * n));
        for (int b = 0; b < n; ++b) {
          const uint32_t dst = smem_u32(smem + (size_t)slot * kSlotBytes<kTokens> + (size_t)b * kStage);
          const int c = (kb + b) * kRowBytes;
          tma_load_3d_pair(dst, &map_w, c, n0, w.e, bar);
          if (!a.rows) tma_load_2d_pair(dst + kABytes, &map_x, c, w.row0 + mine, bar);
        }
        if (++slot == kNSlots) { slot = 0; phase ^= 1u; }
      }
    }
    // Every copy is read by a product that the epilogue waits for.  Where a wait ran out, copies may be on their way that nobody
    // waits for, counted on the partner's barrier: they get the time of a thousand copies.
    if (*abort_flag && polls != 0) {
      const unsigned long long t0 = global_ns();
      while (global_ns() - t0 < 5000000ull) {}
    }
    }
    __syncwarp();
  } else if (warp == 1) {
    if (lane == 0 && rank == 0) {
      int slot = 0;
      uint32_t phase = 0, pass = 0;
      bool ok = true;
      const uint32_t empty0 = map_to_rank(smem_u32(&ctl->empty[0]), 0), empty1 = map_to_rank(smem_u32(&ctl->empty[0]), 1);
      const uint32_t done0 = map_to_rank(smem_u32(&ctl->tmem_full[0]), 0), done1 = map_to_rank(smem_u32(&ctl->tmem_full[0]), 1);
      for (Walk w(plan, a.experts, (uint32_t)feature_tiles); ok && w.valid(); w.next(), ++pass) {
        const uint32_t buf = pass & 1u, d = tmem_base + buf * (uint32_t)kTokens;
        if (!(ok = wait_for(smem_u32(&ctl->tmem_empty[buf]), ((pass >> 1) & 1u) ^ 1u, abort_flag, polls))) break;
        tc_fence_after();
        for (int kb = 0; kb < blocks; kb += kSub) {
          if (!(ok = wait_for(smem_u32(&ctl->full[slot]), phase, abort_flag, polls))) break;
          tc_fence_after();
          const uint32_t at = smem_u32(smem + (size_t)slot * kSlotBytes<kTokens>);
          const int n = min(kSub, blocks - kb);
          for (int b = 0; b < n; ++b) {
            const uint64_t adesc = smem_desc_sw128(at + (uint32_t)(b * kStage)), bdesc = smem_desc_sw128(at + (uint32_t)(b * kStage + kABytes));
#pragma unroll
            for (int j = 0; j < kRowBytes / 32; ++j)
              mma<kInt, 2>(d, adesc + (uint64_t)(2 * j), bdesc + (uint64_t)(2 * j), idesc, kb > 0 || b > 0 || j > 0);
          }
          mma_commit_pair(empty0 + 8u * (uint32_t)slot);
          mma_commit_pair(empty1 + 8u * (uint32_t)slot);
          if (++slot == kNSlots) { slot = 0; phase ^= 1u; }
        }
        if (!ok) break;
        mma_commit_pair(done0 + 8u * buf);
        mma_commit_pair(done1 + 8u * buf);
      }
      // The products are over before the memory that they use is given back, whoever gave up waiting for them.
      mma_commit_pair(map_to_rank(smem_u32(&ctl->drained), 0));
      wait_quiet(smem_u32(&ctl->drained), 0);
    }
    __syncwarp();
  } else if (warp >= 4 + kEpiWarps) {
    // Rows by a list: 16-byte copies, eight lanes to a row of 128 bytes (a tensor copy of four listed rows takes 65 clocks, three
    // times what the tensor cores leave: 8192 rows x 2048 x 8192 over 16 experts 316 us, with these copies @@ us).
    constexpr int kPer = kHalfRows * 8 / (32 * kGatherWarps);      // copies per thread and block of K
    const int u = threadIdx.x - 32 * (4 + kEpiWarps), part = u & 7;
    const int64_t row_bytes = a.K * (kInt ? 1 : 2);
    const char* x = reinterpret_cast<const char*>(a.x);
    int slot = 0;
    uint32_t phase = 0;
    bool ok = true;
    for (Walk w(plan, a.experts, (uint32_t)feature_tiles); ok && w.valid(); w.next()) {
      w.locate(kTokens);
      const char* from[kPer];
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int row = (int)rank * kHalfRows + i * 4 * kGatherWarps + (u >> 3);
        from[i] = x + (int64_t)source_row(a, w.row0 + min(row, w.rows - 1)) * a.ld_x * (kInt ? 1 : 2) + part * 16;
      }
      for (int kb = 0; kb < blocks; kb += kSub) {
        const int n = min(kSub, blocks - kb);
        if (lane == 0) ok = wait_for(smem_u32(&ctl->empty[slot]), phase ^ 1u, abort_flag, polls);
        ok = __shfl_sync(0xFFFFFFFFu, ok, 0);
        if (!ok) break;
        for (int b = 0; b < n; ++b) {
          const uint32_t dst = smem_u32(smem + (size_t)slot * kSlotBytes<kTokens> + (size_t)b * kStage + kABytes);
          const int64_t at = (int64_t)(kb + b) * kRowBytes;
          const uint32_t bytes = at + part * 16 < row_bytes ? 16u : 0u;       // behind the row: zeros
          const int64_t skip = bytes ? at : 0;
#pragma unroll
          for (int i = 0; i < kPer; ++i) {
            const int row = i * 4 * kGatherWarps + (u >> 3);
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst + (uint32_t)(row * kRowBytes + ((part ^ (row & 7)) << 4))),
                         "l"(from[i] + skip), "r"(bytes) : "memory");
          }
        }
        asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(&ctl->gathered[slot])) : "memory");
        if (++slot == kNSlots) { slot = 0; phase ^= 1u; }
      }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
  } else if (warp == 3) {
    // Rows by a list: hands the copies of a slot over to the tensor cores' side of memory and reports them.
    if (lane == 0 && a.rows) {
      int slot = 0;
      uint32_t phase = 0;
      bool ok = true;
      const uint32_t full0 = map_to_rank(smem_u32(&ctl->full[0]), 0);
      for (Walk w(plan, a.experts, (uint32_t)feature_tiles); ok && w.valid(); w.next()) {
        for (int kb = 0; kb < blocks; kb += kSub) {
          if (!(ok = wait_for(smem_u32(&ctl->gathered[slot]), phase, abort_flag, polls))) break;
          fence_proxy_async_smem();
          mbar_arrive_cluster(full0 + 8u * (uint32_t)slot);
          if (++slot == kNSlots) { slot = 0; phase ^= 1u; }
        }
      }
    }
    __syncwarp();
  } else if (warp >= 4) {
    const int quarter = warp & 3, half = (warp - 4) >> 2;
    const int f = quarter * 32 + lane, c0 = half * kHalfRows;        // feature of this CTA, first row of the tile
    float* x_scale = ctl->x_scale[warp - 4];
    TY* y = reinterpret_cast<TY*>(a.y);
    const TY* res = reinterpret_cast<const TY*>(a.residual);
    bool ok = !*abort_flag;
    uint32_t pass = 0;
    const uint32_t release = map_to_rank(smem_u32(&ctl->tmem_empty[0]), 0);
    for (Walk w(plan, a.experts, (uint32_t)feature_tiles); w.valid(); w.next(), ++pass) {
      w.locate(kTokens);
      const uint32_t buf = pass & 1u;
      const int n = w.f * kPairFeatures + (int)rank * kHalf + f;
      const Feature<TY> feature(a, w.e, n);
      if (kInt) {
        __syncwarp();
        for (int j = lane; j < kHalfRows; j += 32)
          x_scale[j] = a.x_scale && c0 + j < w.rows ? a.x_scale[source_row(a, w.row0 + c0 + j)] : 1.f;
        __syncwarp();
      }
      if (ok) {
        if (lane == 0) ok = wait_for(smem_u32(&ctl->tmem_full[buf]), (pass >> 1) & 1u, abort_flag, polls);
        ok = __shfl_sync(0xFFFFFFFFu, ok, 0);
      }
      tc_fence_after();
      const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16) + buf * (uint32_t)kTokens;
#pragma unroll 1
      for (int c = c0; c < c0 + kHalfRows && c < w.rows; c += 32) {
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
        float v[32];
#pragma unroll
        for (int j = 0; j < 32; j += 4) {
          const float4 s = kInt ? *reinterpret_cast<const float4*>(x_scale + (c - c0) + j) : make_float4(1.f, 1.f, 1.f, 1.f);
          v[j] = feature.finish(a, sum_value<kInt>(r[j]), s.x);
          v[j + 1] = feature.finish(a, sum_value<kInt>(r[j + 1]), s.y);
          v[j + 2] = feature.finish(a, sum_value<kInt>(r[j + 2]), s.z);
          v[j + 3] = feature.finish(a, sum_value<kInt>(r[j + 3]), s.w);
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
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_cluster(release + 8u * buf);
    }
  }

  tc_fence_before();
  __syncthreads();
  cluster_sync_all();                                // the partner no longer touches this CTA's memory
  if (warp == 2) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(kTmemCols) : "memory");
  }
}

template <int kTokens, bool kInt, typename TY>
cudaError_t launch(const MatmulArgs& a, cudaStream_t s) {
  const int es = kInt ? 1 : 2;
  const int64_t feature_tiles = (a.N + kPairFeatures - 1) / kPairFeatures;
  int64_t token_tiles = (a.R + kTokens - 1) / kTokens;
  if (a.offsets) token_tiles = a.R / kTokens + (a.experts < a.R ? a.experts : a.R);    // at most: one that is not full per expert
  const int64_t tiles = token_tiles * feature_tiles;
  if (tiles > 0x7FFFFFFF) return cudaErrorInvalidValue;
  CUtensorMap map_w, map_x;
  const int box_n = a.N < kHalf ? (int)a.N : kHalf, box_t = a.x_rows < kTokens / 2 ? (int)a.x_rows : kTokens / 2;
  cudaError_t e = encode_weights(&map_w, a, box_n);
  if (e == cudaSuccess) e = encode_rows(&map_x, a.x, a.K * es, a.x_rows, a.ld_x * es, box_t);
  if (e != cudaSuccess) return e;
  const int tx = (box_n + (a.rows ? 0 : box_t)) * kRowBytes;
  const unsigned threads = kThreads + (a.rows ? 32 * kGatherWarps : 0);
  const auto kern = matmul_wide_kernel<kTokens, kInt, TY>;
  // Clusters that the device holds at once; 0 until the kernel is set up there.  Devices beyond the table are set up on every call.
  static std::atomic<int> resident[64];
  int dev = 0;
  if ((e = cudaGetDevice(&dev)) != cudaSuccess) return e;
  int cap = dev < 64 ? resident[dev].load(std::memory_order_acquire) : 0;
  if (cap == 0) {
    const size_t most = smem_bytes<kTokens>(kMaxExperts);
    if ((e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most)) != cudaSuccess) return e;
    if ((e = max_clusters(kern, 2, kThreads + 32 * kGatherWarps, most, &cap)) != cudaSuccess) return e;
    if (cap < 1) return cudaErrorInvalidConfiguration;
    if (dev < 64) resident[dev].store(cap, std::memory_order_release);
  }
  const int64_t clusters = tiles < cap ? tiles : cap;
  const long long polls = g_debug_wait_polls.load(std::memory_order_relaxed);
  return launch_pdl(kern, dim3((unsigned)(2 * clusters)), threads, smem_bytes<kTokens>(a.experts), s, map_w, map_x, a,
                    instr_desc(a.operand, kPairFeatures, kTokens), (int)feature_tiles, tx, polls);
}

template <int kTokens>
cudaError_t launch_type(const MatmulArgs& a, cudaStream_t s) {
  const bool whole = a.operand == BL_I8;
  switch (a.yt) {
    case BL_F32: return whole ? launch<kTokens, true, float>(a, s) : launch<kTokens, false, float>(a, s);
    case BL_F16: return whole ? launch<kTokens, true, __half>(a, s) : launch<kTokens, false, __half>(a, s);
    default: return whole ? launch<kTokens, true, __nv_bfloat16>(a, s) : launch<kTokens, false, __nv_bfloat16>(a, s);
  }
}

}  // namespace

cudaError_t launch_matmul_wide(const MatmulArgs& a, int tokens, cudaStream_t s) {
  return tokens == 128 ? launch_type<128>(a, s) : launch_type<256>(a, s);
}

}  // namespace bl
