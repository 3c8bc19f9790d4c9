// 8-bit (and fp16, bf16) matrix products of few rows: decode steps and short lists of rows.  Bound by the weights' bytes.
// A tile is 128 output features x kTokens rows.  Where that leaves SMs without work, a cluster of `splits` CTAs shares the K axis of a
// tile and joins its sums through shared memory (whole numbers exactly, fp32 in the order of the CTAs); there is a cluster per
// tile then.  Without, the grid is persistent: loads run ahead from tile to tile, and two accumulators take turns.
// A ring slot holds `sub` blocks of 128 bytes of K.  Where K is a whole number of blocks one tensor copy brings the weights of
// a slot, and one the tokens: a copy costs about 70 clocks and 3.4 per row of 128 bytes (measured on one SM), so small
// ones are dear.  Without lists it is known at once which weights come first: those of a ring are brought into L2 while the kernel
// before this one on the stream still runs, and copied from there in the stream's order, so that weights may be written just before.
// Warp 0 loads (tokens four rows at a time where a list says which), warp 1 multiplies, warps 2-5 take a quarter of the lanes
// each to y.  Waits are bounded; a tile whose wait runs out is written as NaN.
#include "matmul_common.cuh"

namespace bl {

namespace {

using namespace mm;

constexpr int kThreads = 192;
constexpr int kFeatures = 128;              // of a tile: rows of weights per instruction
constexpr int kWBlock = kFeatures * kRowBytes;
constexpr int kMaxSlots = 8;

struct Control {
  unsigned long long full[kMaxSlots], empty[kMaxSlots], done[2], taken[2], drained;
  uint32_t tmem_base;
  int abort_flag, peer_abort;
  alignas(16) float x_scale[4][64];
};

// How a launch cuts its work and its shared memory.
struct Cut {
  int feature_tiles, splits, sub, slots, packed;   // packed: a slot's weights come in one copy, its tokens in another
  int x_block;                                     // bytes of a block of tokens: of those that there can be, in eights
  int w_bytes, x_bytes;                            // of a copy
  int behind;                                      // bytes that an instruction may read behind the last slot: tokens that there are not
  uint32_t idesc;
};

template <int kTokens, bool kInt, typename TY>
__global__ void __launch_bounds__(kThreads)
matmul_narrow_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x, MatmulArgs a, Cut cut, long long polls) {
  constexpr int kCols = 2 * kTokens;                          // of tensor memory: two accumulators
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  const int splits = cut.splits, sub = cut.sub, slots = cut.slots;
  const int slot_bytes = sub * (kWBlock + cut.x_block);
  // slots, then room for what an instruction reads behind the last one, then the other CTAs' sums [CTA][token of mine][feature]
  uint32_t* parts = reinterpret_cast<uint32_t*>(smem + slots * slot_bytes + cut.behind);
  Control* ctl = reinterpret_cast<Control*>(reinterpret_cast<unsigned char*>(parts) + (splits > 1 ? kTokens * kFeatures * 4 : 0));
  int* plan = reinterpret_cast<int*>(ctl + 1);
  volatile int* abort_flag = &ctl->abort_flag;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = splits > 1 ? (int)(blockIdx.x % (unsigned)splits) : 0;
  const uint32_t item = blockIdx.x / (uint32_t)splits, items = gridDim.x / (uint32_t)splits;
  const int es = kInt ? 1 : 2;
  const int blocks = (int)((a.K * es + kRowBytes - 1) / kRowBytes);
  const int steps = (blocks + sub - 1) / sub;                // slots' worth of K; this CTA's:
  const int s0 = (int)((int64_t)steps * rank / splits), s1 = (int)((int64_t)steps * (rank + 1) / splits);
  auto copies = [&](int step) { return cut.packed ? 1 : min(sub, blocks - step * sub); };
  if (threadIdx.x == 0) {
    prefetch_map(&map_w);
    prefetch_map(&map_x);
    for (int s = 0; s < slots; ++s) { mbar_init(smem_u32(&ctl->full[s]), 1); mbar_init(smem_u32(&ctl->empty[s]), 1); }
    for (int b = 0; b < 2; ++b) { mbar_init(smem_u32(&ctl->done[b]), 1); mbar_init(smem_u32(&ctl->taken[b]), 4); }
    mbar_init(smem_u32(&ctl->drained), 1);
    ctl->abort_flag = polls == 0;
    ctl->peer_abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    if (!a.offsets && polls != 0) {
      // one expert: the feature tile of the first tile of this CTA
      const int row_tiles = (int)((a.R + kTokens - 1) / kTokens), first_n0 = (int)(item / (uint32_t)row_tiles) * kFeatures;
      for (int step = s0; step < min(s0 + slots, s1); ++step) {
        if (cut.packed) {
          tma_prefetch_4d(&map_w, 0, first_n0, step * sub, 0);
        } else {
          for (int b = 0; b < sub && step * sub + b < blocks; ++b) tma_prefetch_4d(&map_w, (step * sub + b) * kRowBytes, first_n0, 0, 0);
        }
      }
    }
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ctl->tmem_base)), "r"(kCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    pdl_launch_dependents();                       // not before the tensor memory is ours: a kernel behind this one may take some, then wait for this one
  }
  __syncwarp();
  if (a.offsets) pdl_wait();
  if (warp == 2) make_plan(a, plan, kTokens);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (splits > 1) asm volatile("barrier.cluster.arrive.release;" ::: "memory");      // this CTA is there: its memory may be written
  const uint32_t tmem_base = ctl->tmem_base;
  if (!a.offsets) pdl_wait();                        // so far nothing that the kernel before could have written was read
  const Walk from(plan, a.experts, cut.feature_tiles, item, items);
  const int quarter = warp & 3, f = quarter * 32 + lane;
  const bool writer = warp >= 2;
  TY* y = reinterpret_cast<TY*>(a.y);
  const TY* res = reinterpret_cast<const TY*>(a.residual);
  // What a warp needs of a tile before its sums are there.
  auto take_scales = [&](const Walk& w) {
    __syncwarp();
    for (int j = lane; j < kTokens; j += 32) ctl->x_scale[quarter][j] = a.x_scale && j < w.rows ? a.x_scale[source_row(a, w.row0 + j)] : 1.f;
    __syncwarp();
  };
  // Sums of up to kN rows on their way out, without a branch between them: their loads and conversions overlap.
  auto put = [&](const Feature<TY>& feature, int64_t row, int n, int rows, const auto& sums, const float* x_scale, bool good) {
    constexpr int kN = sizeof(sums) / sizeof(sums[0]);
    Raw<TY> add[kN];
    if (res) {
      const TY* r = res + row * a.ld_res + n;
#pragma unroll
      for (int j = 0; j < kN; ++j) add[j] = load_raw(r + min(j, rows - 1) * a.ld_res);
    }
    float v[kN];
#pragma unroll
    for (int j = 0; j < kN; j += 2) feature.finish2(sum_value<kInt>(sums[j]), sum_value<kInt>(sums[j + 1]), x_scale[j], x_scale[j + 1], v[j], v[j + 1]);
    if (!good) {
#pragma unroll
      for (int j = 0; j < kN; ++j) v[j] = __uint_as_float(0x7FC00000u);
    }
    if (res) {
#pragma unroll
      for (int j = 0; j < kN; ++j) v[j] += raw_value<TY>(add[j]);
    }
    TY* out = y + row * a.ld_y + n;
    if (rows >= kN) {
#pragma unroll
      for (int j = 0; j < kN; ++j) out[j * a.ld_y] = out_cast<TY>(v[j]);
    } else {
#pragma unroll
      for (int j = 0; j < kN; ++j)
        if (j < rows) out[j * a.ld_y] = out_cast<TY>(v[j]);
    }
  };

  int issued = 0;                                            // slots that thread 0 filled
  if (warp == 0) {
    int slot = 0;
    uint32_t phase = 0;
    bool ok = polls != 0;
    for (Walk w = from; ok && w.valid(); w.next()) {
      w.locate(kTokens);
      const int n0 = w.f * kFeatures;
      // Listed rows four at a time, as many as there are (places behind them hold what was there, and nobody reads their sums).
      const int fours = (w.rows + 3) / 4;
      int r[4] = {0, 0, 0, 0};
      if (a.rows && lane < fours) {
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = source_row(a, w.row0 + min(4 * lane + i, w.rows - 1));
      }
      for (int step = s0; step < s1; ++step) {
        const uint32_t bar = smem_u32(&ctl->full[slot]);
        if (lane == 0) {
          ok = mbar_wait_polls(smem_u32(&ctl->empty[slot]), phase ^ 1u, abort_flag, polls);
          if (ok) {
            const int x_bytes = a.rows ? fours * 4 * kRowBytes * min(sub, blocks - step * sub) : cut.x_bytes * copies(step);
            mbar_arrive_expect_tx(bar, (uint32_t)(x_bytes + cut.w_bytes * copies(step)));
            const uint32_t dst = smem_u32(smem + slot * slot_bytes);
            if (cut.packed) {
              tma_load_4d(dst, &map_w, 0, n0, step * sub, w.e, bar);
            } else {
              for (int b = 0; b < sub && step * sub + b < blocks; ++b) tma_load_4d(dst + b * kWBlock, &map_w, (step * sub + b) * kRowBytes, n0, 0, w.e, bar);
            }
          }
        }
        if (a.rows) ok = __shfl_sync(0xFFFFFFFFu, ok, 0);
        if (!ok || (!a.rows && lane != 0)) break;
        const uint32_t dst = smem_u32(smem + slot * slot_bytes) + (uint32_t)(sub * kWBlock);
        if (!a.rows && cut.packed) {
          tma_load_3d(dst, &map_x, 0, w.row0, step * sub, bar);
        } else {
          for (int b = 0; b < sub && step * sub + b < blocks; ++b) {
            const int c = (step * sub + b) * kRowBytes;
            if (!a.rows) tma_load_3d(dst + b * cut.x_block, &map_x, c, w.row0, 0, bar);
            else if (lane < fours) tma_gather4(dst + b * cut.x_block + lane * 4 * kRowBytes, &map_x, c, r, bar);
          }
        }
        ++issued;
        if (++slot == slots) { slot = 0; phase ^= 1u; }
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    if (lane == 0) {
      int slot = 0;
      uint32_t phase = 0, pass = 0;
      bool ok = polls != 0;
      for (Walk w = from; ok && w.valid(); w.next(), ++pass) {
        const uint32_t buf = pass & 1u, d = tmem_base + buf * (uint32_t)kTokens;
        if (!(ok = mbar_wait_polls(smem_u32(&ctl->taken[buf]), ((pass >> 1) & 1u) ^ 1u, abort_flag, polls))) break;
        tc_fence_after();
        for (int step = s0; step < s1; ++step) {
          if (!(ok = mbar_wait_polls(smem_u32(&ctl->full[slot]), phase, abort_flag, polls))) break;
          tc_fence_after();
          const uint32_t at = smem_u32(smem + slot * slot_bytes);
          for (int b = 0; b < sub && step * sub + b < blocks; ++b) {
            const uint64_t adesc = smem_desc_sw128(at + (uint32_t)(b * kWBlock)), bdesc = smem_desc_sw128(at + (uint32_t)(sub * kWBlock + b * cut.x_block));
#pragma unroll
            for (int j = 0; j < kRowBytes / 32; ++j)
              mma<kInt, 1>(d, adesc + (uint64_t)(2 * j), bdesc + (uint64_t)(2 * j), cut.idesc, step > s0 || b > 0 || j > 0);
          }
          mma_commit(smem_u32(&ctl->empty[slot]));
          if (++slot == slots) { slot = 0; phase ^= 1u; }
        }
        if (ok) mma_commit(smem_u32(&ctl->done[buf]));
      }
      // The products are over before this CTA gives its memory back, whoever gave up waiting for them.
      mma_commit(smem_u32(&ctl->drained));
      mbar_wait_quiet(smem_u32(&ctl->drained), 0);
    }
    __syncwarp();
  } else if (splits == 1) {
    bool ok = polls != 0;
    uint32_t pass = 0;
    for (Walk w = from; w.valid(); w.next(), ++pass) {
      w.locate(kTokens);
      const uint32_t buf = pass & 1u;
      const int n = w.f * kFeatures + f;
      const Feature<TY> feature(a, w.e, n);
      take_scales(w);
      if (ok) {
        if (lane == 0) ok = mbar_wait_polls(smem_u32(&ctl->done[buf]), (pass >> 1) & 1u, abort_flag, polls);
        ok = __shfl_sync(0xFFFFFFFFu, ok, 0);
      }
      tc_fence_after();
      const uint32_t taddr = tmem_base + buf * (uint32_t)kTokens + ((uint32_t)(quarter * 32) << 16);
#pragma unroll 1
      for (int c = 0; c < kTokens && c < w.rows; c += 16) {
        uint32_t r[16];
        tmem_ld16(taddr + (uint32_t)c, r);
        if (feature.on) put(feature, w.row0 + c, n, w.rows - c, r, ctl->x_scale[quarter] + c, ok);
      }
      // One that gave up reports nothing more: its report would stand for a warp that still reads, and the next products would go over
      // what that one reads.  The multiplying warp gives up as well then, and every tile from here on is NaN.
      tc_fence_before();
      __syncwarp();
      if (ok && lane == 0) mbar_arrive(smem_u32(&ctl->taken[buf]));
    }
  }

  if (splits > 1) {
    // One tile for the cluster, if any; every thread of it takes part in its barriers.
    asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
    const int shift = __ffs(kTokens / splits) - 1, each = 1 << shift;      // tokens that a CTA finishes
    Walk w = from;
    const bool mine = writer && w.valid();
    if (w.valid()) w.locate(kTokens);
    const int n = w.f * kFeatures + f;
    const Feature<TY> feature(a, w.e, mine ? n : (int)a.N);
    if (mine) {
      take_scales(w);
      bool ok = polls != 0;
      if (ok) {
        if (lane == 0) ok = mbar_wait_polls(smem_u32(&ctl->done[0]), 0, abort_flag, polls);
        ok = __shfl_sync(0xFFFFFFFFu, ok, 0);
      }
      tc_fence_after();
#pragma unroll 1
      for (int c = 0; c < kTokens && c < w.rows; c += 16) {
        uint32_t r[16];
        tmem_ld16(tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)c, r);
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const int token = c + j, owner = token >> shift;
          if (token < w.rows) st_cluster(map_to_rank(smem_u32(parts + ((rank << shift) + (token & (each - 1))) * kFeatures + f), (uint32_t)owner), r[j]);
        }
      }
      if (!ok && lane == 0)
        for (int o = 0; o < splits; ++o) st_cluster(map_to_rank(smem_u32(&ctl->peer_abort), (uint32_t)o), 1u);
    }
    asm volatile("barrier.cluster.arrive.release;\nbarrier.cluster.wait.acquire;" ::: "memory");
    if (mine && feature.on) {
      const bool bad = *reinterpret_cast<volatile int*>(&ctl->peer_abort) != 0;
      const int t0 = rank << shift, here = min(each, w.rows - t0);
#pragma unroll 1
      for (int j = 0; j < here; j += 8) {
        uint32_t sums[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int at = min(j + i, here - 1);
          sums[i] = parts[at * kFeatures + f];
#pragma unroll
          for (int s = 1; s < 8; ++s) {
            if (s < splits) {
              const uint32_t v = parts[((s << shift) + at) * kFeatures + f];
              sums[i] = kInt ? sums[i] + v : __float_as_uint(__uint_as_float(sums[i]) + __uint_as_float(v));
            }
          }
        }
        put(feature, w.row0 + t0 + j, n, here - j, sums, ctl->x_scale[quarter] + t0 + j, !bad);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  // Where a wait ran out, whichever role's and however late, copies may be on their way that nobody waits for any more: they must not
  // land in a CTA that is gone.  Now that every role is through, thread 0 waits for the last round of the ring; those before it were
  // waited for to fill the slots again.
  if (threadIdx.x == 0 && *abort_flag)
    for (int i = max(0, issued - slots); i < issued; ++i) mbar_wait_quiet(smem_u32(&ctl->full[i % slots]), (uint32_t)(i / slots & 1));
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(kCols) : "memory");
  }
}

template <int kTokens, bool kInt, typename TY>
cudaError_t launch(const MatmulArgs& a, int splits, int per_sm, cudaStream_t s) {
  const int es = kInt ? 1 : 2;
  const int64_t blocks = (a.K * es + kRowBytes - 1) / kRowBytes;
  const int64_t feature_tiles = (a.N + kFeatures - 1) / kFeatures;
  int64_t token_tiles = (a.R + kTokens - 1) / kTokens;
  if (a.offsets) token_tiles = a.R / kTokens + (a.experts < a.R ? a.experts : a.R);    // at most: one that is not full per expert
  if (token_tiles * feature_tiles * splits > 0x7FFFFFFF) return cudaErrorInvalidValue;
  // Slots of up to four blocks of K, as many as leave room for three slots at least.
  Cut cut;
  const int box_t = a.rows || a.x_rows > kTokens - 8 ? kTokens : ((int)a.x_rows + 7) / 8 * 8;
  const int block = (kFeatures + box_t) * kRowBytes;
  cut.x_block = box_t * kRowBytes;
  cut.behind = (kTokens - box_t) * kRowBytes;
  const int budget = (227 - per_sm) * 1024 / per_sm;          // an SM's shared memory, less what the system keeps per CTA
  const int fixed = 1024 + (int)sizeof(Control) + (int)plan_bytes(a.experts) + cut.behind + (splits > 1 ? kTokens * kFeatures * 4 : 0);
  cut.sub = 4;
  while (cut.sub > 1 && (budget - fixed) / (cut.sub * block) < 3) cut.sub /= 2;
  cut.slots = (budget - fixed) / (cut.sub * block);
  if (cut.slots > kMaxSlots) cut.slots = kMaxSlots;
  cut.feature_tiles = (int)feature_tiles;
  while (splits > 1 && (blocks + cut.sub - 1) / cut.sub < splits) splits /= 2;       // no CTA without a slot's worth of K
  cut.splits = splits;
  cut.packed = a.K * es % kRowBytes == 0;
  cut.w_bytes = kWBlock * (cut.packed ? cut.sub : 1);
  cut.x_bytes = box_t * kRowBytes * (cut.packed ? cut.sub : 1);
  cut.idesc = instr_desc(a.operand, kFeatures, (box_t + 15) / 16 * 16);
  CUtensorMap map_w, map_x;
  cudaError_t e = encode_blocks(&map_w, a.w, a.K * es, a.N, a.ld_w * es, a.experts, a.expert_stride * es, kFeatures, cut.packed ? cut.sub : 0);
  if (e != cudaSuccess) return e;
  if (a.rows) e = encode_rows(&map_x, a.x, a.K * es, a.x_rows, a.ld_x * es, 1);
  else e = encode_blocks(&map_x, a.x, a.K * es, a.x_rows, a.ld_x * es, 0, 0, box_t, cut.packed ? cut.sub : 0);
  if (e != cudaSuccess) return e;
  const auto kern = matmul_narrow_kernel<kTokens, kInt, TY>;
  static std::atomic<uint64_t> ready{0};                     // devices on which the kernel's shared memory limit is set
  int dev = 0;
  if ((e = cudaGetDevice(&dev)) != cudaSuccess) return e;
  if (dev > 63 || !(ready.load(std::memory_order_acquire) >> dev & 1)) {
    if ((e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, 226 * 1024)) != cudaSuccess) return e;
    if (dev <= 63) ready.fetch_or(1ull << dev, std::memory_order_acq_rel);
  }
  int sms = 0;
  if ((e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev)) != cudaSuccess) return e;
  int64_t clusters = token_tiles * feature_tiles;
  if (splits == 1 && clusters > (int64_t)sms * per_sm) clusters = (int64_t)sms * per_sm;
  const size_t smem = (size_t)fixed + (size_t)cut.slots * cut.sub * block;
  const long long polls = g_debug_wait_polls.load(std::memory_order_relaxed);
  return launch_pdl_clusters(kern, dim3((unsigned)(clusters * splits)), splits > 1 ? (unsigned)splits : 0u, kThreads, smem, s, map_w, map_x, a, cut, polls);
}

template <int kTokens>
cudaError_t launch_type(const MatmulArgs& a, int splits, int per_sm, cudaStream_t s) {
  const bool whole = a.operand == BL_I8;
  switch (a.yt) {
    case BL_F32: return whole ? launch<kTokens, true, float>(a, splits, per_sm, s) : launch<kTokens, false, float>(a, splits, per_sm, s);
    case BL_F16: return whole ? launch<kTokens, true, __half>(a, splits, per_sm, s) : launch<kTokens, false, __half>(a, splits, per_sm, s);
    default: return whole ? launch<kTokens, true, __nv_bfloat16>(a, splits, per_sm, s) : launch<kTokens, false, __nv_bfloat16>(a, splits, per_sm, s);
  }
}

}  // namespace

cudaError_t launch_matmul_narrow(const MatmulArgs& a, int tokens, int splits, int per_sm, cudaStream_t s) {
  return tokens == 16 ? launch_type<16>(a, splits, per_sm, s) : tokens == 32 ? launch_type<32>(a, splits, per_sm, s)
                                                                               : launch_type<64>(a, splits, per_sm, s);
}

}  // namespace bl
