// 8-bit (and fp16, bf16) matrix products of few rows: decode steps and short lists of rows.  Bound by the weights' bytes.
// A tile is 128 output features x kTokens rows; a cluster of `splits` CTAs shares the K axis of one tile, so that the loads
// of few tiles spread over the GPU, and joins its sums through shared memory (the whole numbers exactly, fp32 in the order of the
// CTAs).  One tile per cluster: what a CTA spends on its start and its end is covered by the others on the SM.
// Warp 0 loads (weights as boxes of 128 rows x 128 bytes; tokens as boxes, or four rows at a time where a list says which),
// warp 1 multiplies, warps 2-5 take a quarter of the lanes each to y.
// Waits are bounded; a tile whose wait runs out is written as NaN.
#include "matmul_common.cuh"

namespace bl {

namespace {

using namespace mm;

constexpr int kThreads = 192;
constexpr int kFeatures = 128;
constexpr int kABytes = kFeatures * kRowBytes;
constexpr int kMaxSlots = 8;
constexpr size_t kBudget = 113 * 1024;      // two CTAs per SM

struct Control {
  unsigned long long full[kMaxSlots], empty[kMaxSlots], done, drained;
  uint32_t tmem_base;
  int abort_flag, peer_abort;
  Tile tile;
  float x_scale[64];
};

template <int kTokens>
__host__ __device__ constexpr int slots_for(bool join) {
  const size_t n = (kBudget - 1024 - sizeof(Control) - (join ? (size_t)kTokens * kFeatures * 4 : 0)) / (kABytes + kTokens * kRowBytes);
  return n > kMaxSlots ? kMaxSlots : (int)n;
}
template <int kTokens>
constexpr size_t smem_bytes(bool join) {
  return 1024 + (size_t)slots_for<kTokens>(join) * (kABytes + kTokens * kRowBytes) + (join ? (size_t)kTokens * kFeatures * 4 : 0) + sizeof(Control);
}

template <int kTokens, bool kInt, typename TY>
__global__ void __launch_bounds__(kThreads)
matmul_narrow_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x, MatmulArgs a, uint32_t idesc,
                     int feature_tiles, int splits, int tx_bytes, long long polls) {
  constexpr int kStage = kABytes + kTokens * kRowBytes;
  constexpr int kCols = kTokens < 32 ? 32 : kTokens;          // of tensor memory
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  const int slots = splits > 1 ? slots_for<kTokens>(true) : slots_for<kTokens>(false);
  uint32_t* parts = reinterpret_cast<uint32_t*>(smem + (size_t)slots * kStage);      // [CTA][token of mine][feature]
  Control* ctl = reinterpret_cast<Control*>(reinterpret_cast<unsigned char*>(parts) + (splits > 1 ? (size_t)kTokens * kFeatures * 4 : 0));
  volatile int* abort_flag = &ctl->abort_flag;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = splits > 1 ? (int)(blockIdx.x % (unsigned)splits) : 0;
  const unsigned item = blockIdx.x / (unsigned)splits;
  pdl_launch_dependents();
  if (threadIdx.x == 0) {
    prefetch_map(&map_w);
    prefetch_map(&map_x);
    for (int s = 0; s < slots; ++s) { mbar_init(smem_u32(&ctl->full[s]), 1); mbar_init(smem_u32(&ctl->empty[s]), 1); }
    mbar_init(smem_u32(&ctl->done), 1);
    mbar_init(smem_u32(&ctl->drained), 1);
    ctl->abort_flag = polls == 0;
    ctl->peer_abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ctl->tmem_base)), "r"(kCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  pdl_wait();
  const int n0 = (int)(item % (unsigned)feature_tiles) * kFeatures;
  if (warp == 2) {
    const Tile t = find_tile(a, (int)(item / (unsigned)feature_tiles), kTokens);
    if (lane == 0) ctl->tile = t;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (splits > 1) asm volatile("barrier.cluster.arrive.release;" ::: "memory");      // this CTA is there: its memory may be written
  const Tile tile = ctl->tile;
  const uint32_t tmem_base = ctl->tmem_base;
  const int es = kInt ? 1 : 2;
  const int blocks = (int)((a.K * es + kRowBytes - 1) / kRowBytes);
  const int kb0 = (int)((int64_t)blocks * rank / splits), kb1 = (int)((int64_t)blocks * (rank + 1) / splits);

  if (tile.rows == 0 || *abort_flag) {
    // no such tile (the whole cluster sees the same), or no waits allowed
  } else if (warp == 0) {
    int r[4] = {0, 0, 0, 0};
    if (a.rows && lane < kTokens / 4) {
#pragma unroll
      for (int i = 0; i < 4; ++i) r[i] = source_row(a, tile.row0 + min(4 * lane + i, tile.rows - 1));
    }
    int slot = 0;
    uint32_t phase = 0;
    int kb = kb0;
    for (; kb < kb1; ++kb) {
      bool ok = true;
      if (lane == 0) {
        ok = wait_for(smem_u32(&ctl->empty[slot]), phase ^ 1u, abort_flag, polls);
        if (ok) mbar_arrive_expect_tx(smem_u32(&ctl->full[slot]), (uint32_t)tx_bytes);
      }
      if (!__shfl_sync(0xFFFFFFFFu, ok, 0)) break;
      const uint32_t dst = smem_u32(smem + (size_t)slot * kStage), bar = smem_u32(&ctl->full[slot]);
      if (lane == 0) tma_load_3d(dst, &map_w, kb * kRowBytes, n0, tile.expert, bar);
      if (a.rows) {
        if (lane < kTokens / 4) tma_gather4(dst + kABytes + lane * 4 * kRowBytes, &map_x, kb * kRowBytes, r, bar);
      } else if (lane == 0) {
        tma_load_2d(dst + kABytes, &map_x, kb * kRowBytes, tile.row0, bar);
      }
      if (++slot == slots) { slot = 0; phase ^= 1u; }
    }
    // Copies that nobody waits for any more must not land in a CTA that is gone.
    if (*abort_flag && lane == 0) {
      for (int i = max(kb0, kb - slots); i < kb; ++i)
        wait_quiet(smem_u32(&ctl->full[(i - kb0) % slots]), (uint32_t)((i - kb0) / slots & 1));
    }
  } else if (warp == 1) {
    if (lane == 0) {
      int slot = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int kb = kb0; kb < kb1; ++kb) {
        if (!(ok = wait_for(smem_u32(&ctl->full[slot]), phase, abort_flag, polls))) break;
        tc_fence_after();
        const uint32_t at = smem_u32(smem + (size_t)slot * kStage);
        const uint64_t adesc = smem_desc_sw128(at), bdesc = smem_desc_sw128(at + kABytes);
#pragma unroll
        for (int j = 0; j < kRowBytes / 32; ++j)
          mma<kInt, 1>(tmem_base, adesc + (uint64_t)(2 * j), bdesc + (uint64_t)(2 * j), idesc, kb > kb0 || j > 0);
        mma_commit(smem_u32(&ctl->empty[slot]));
        if (++slot == slots) { slot = 0; phase ^= 1u; }
      }
      // The products are over before this CTA gives its memory back, whoever gave up waiting for them.
      mma_commit(smem_u32(ok ? &ctl->done : &ctl->drained));
      wait_quiet(smem_u32(ok ? &ctl->done : &ctl->drained), 0);
    }
    __syncwarp();
  } else {
    const int e = threadIdx.x - 64;                           // 0..127
    if (e < kTokens) ctl->x_scale[e] = a.x_scale && e < tile.rows ? a.x_scale[source_row(a, tile.row0 + e)] : 1.f;
    asm volatile("bar.sync 1, 128;" ::: "memory");
  }

  if (splits > 1) asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
  const int quarter = warp & 3, f = quarter * 32 + lane, n = n0 + f;
  const bool writer = warp >= 2 && tile.rows > 0;
  TY* y = reinterpret_cast<TY*>(a.y);
  const TY* res = reinterpret_cast<const TY*>(a.residual);
  auto put = [&](const Feature<TY>& feature, int j, float sum) {
    const int64_t row = tile.row0 + j;
    float v = feature.finish(a, sum, ctl->x_scale[j]);
    if (res) v += in_cast(res[row * a.ld_res + n]);
    y[row * a.ld_y + n] = out_cast<TY>(v);
  };
  if (writer) {
    bool ok = !*abort_flag;
    if (ok) {
      if (lane == 0) ok = wait_for(smem_u32(&ctl->done), 0, abort_flag, polls);
      ok = __shfl_sync(0xFFFFFFFFu, ok, 0);
    }
    tc_fence_after();
    const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16);
    if (splits == 1) {
      const Feature<TY> feature(a, tile.expert, n);
#pragma unroll 1
      for (int c = 0; c < kTokens && c < tile.rows; c += 16) {
        uint32_t r[16];
        tmem_ld16(taddr + (uint32_t)c, r);
        if (feature.on) {
#pragma unroll
          for (int j = 0; j < 16; ++j)
            if (c + j < tile.rows) put(feature, c + j, ok ? sum_value<kInt>(r[j]) : __uint_as_float(0x7FC00000u));
        }
      }
    } else {
      const int each = kTokens / splits;                      // tokens that a CTA finishes
#pragma unroll 1
      for (int c = 0; c < kTokens && c < tile.rows; c += 16) {
        uint32_t r[16];
        tmem_ld16(taddr + (uint32_t)c, r);
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const int token = c + j, owner = token / each;
          uint32_t dst;
          asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(dst)
                       : "r"(smem_u32(parts + (rank * each + token - owner * each) * kFeatures + f)), "r"(owner));
          asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(dst), "r"(r[j]) : "memory");
        }
      }
      if (!ok && lane == 0) {
        for (int o = 0; o < splits; ++o) {
          uint32_t dst;
          asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(dst) : "r"(smem_u32(&ctl->peer_abort)), "r"(o));
          asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(dst), "r"(1) : "memory");
        }
      }
    }
  }
  if (splits > 1 && tile.rows > 0) {
    asm volatile("barrier.cluster.arrive.release;\nbarrier.cluster.wait.acquire;" ::: "memory");
    if (writer) {
      const int each = kTokens / splits;
      const bool bad = *reinterpret_cast<volatile int*>(&ctl->peer_abort) != 0;
      const Feature<TY> feature(a, tile.expert, n);
      if (feature.on) {
        for (int j = 0; j < each && rank * each + j < tile.rows; ++j) {
          uint32_t sum = parts[j * kFeatures + f];
          for (int s = 1; s < splits; ++s) {
            const uint32_t v = parts[(s * each + j) * kFeatures + f];
            sum = kInt ? sum + v : __float_as_uint(__uint_as_float(sum) + __uint_as_float(v));
          }
          put(feature, rank * each + j, bad ? __uint_as_float(0x7FC00000u) : sum_value<kInt>(sum));
        }
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(kCols) : "memory");
  }
}

template <int kTokens, bool kInt, typename TY>
cudaError_t launch(const MatmulArgs& a, int splits, cudaStream_t s) {
  const int es = kInt ? 1 : 2;
  const int64_t feature_tiles = (a.N + kFeatures - 1) / kFeatures;
  int64_t token_tiles = (a.R + kTokens - 1) / kTokens;
  if (a.offsets) token_tiles = a.R / kTokens + (a.experts < a.R ? a.experts : a.R);    // at most: one that is not full per expert
  const int64_t grid = token_tiles * feature_tiles * splits;
  if (grid > 0x7FFFFFFF) return cudaErrorInvalidValue;
  CUtensorMap map_w, map_x;
  const int box_n = a.N < kFeatures ? (int)a.N : kFeatures, box_t = a.rows ? 1 : a.x_rows < kTokens ? (int)a.x_rows : kTokens;
  cudaError_t e = encode_weights(&map_w, a, box_n);
  if (e == cudaSuccess) e = encode_rows(&map_x, a.x, a.K * es, a.x_rows, a.ld_x * es, box_t);
  if (e != cudaSuccess) return e;
  const int tx = (box_n + (a.rows ? kTokens : box_t)) * kRowBytes;
  const auto kern = matmul_narrow_kernel<kTokens, kInt, TY>;
  const size_t smem = smem_bytes<kTokens>(splits > 1);
  static std::atomic<uint64_t> ready{0};                     // devices on which the kernel's shared memory limit is set
  int dev = 0;
  if ((e = cudaGetDevice(&dev)) != cudaSuccess) return e;
  if (dev > 63 || !(ready.load(std::memory_order_acquire) >> dev & 1)) {
    const size_t most = smem_bytes<kTokens>(false) > smem_bytes<kTokens>(true) ? smem_bytes<kTokens>(false) : smem_bytes<kTokens>(true);
    if ((e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most)) != cudaSuccess) return e;
    if (dev <= 63) ready.fetch_or(1ull << dev, std::memory_order_acq_rel);
  }
  const long long polls = g_debug_wait_polls.load(std::memory_order_relaxed);
  return launch_pdl_clusters(kern, dim3((unsigned)grid), splits > 1 ? (unsigned)splits : 0u, kThreads, smem, s, map_w, map_x, a,
                             instr_desc(a.operand, kFeatures, kTokens), (int)feature_tiles, splits, tx, polls);
}

template <int kTokens>
cudaError_t launch_type(const MatmulArgs& a, int splits, cudaStream_t s) {
  const bool whole = a.operand == BL_I8;
  switch (a.yt) {
    case BL_F32: return whole ? launch<kTokens, true, float>(a, splits, s) : launch<kTokens, false, float>(a, splits, s);
    case BL_F16: return whole ? launch<kTokens, true, __half>(a, splits, s) : launch<kTokens, false, __half>(a, splits, s);
    default: return whole ? launch<kTokens, true, __nv_bfloat16>(a, splits, s) : launch<kTokens, false, __nv_bfloat16>(a, splits, s);
  }
}

}  // namespace

cudaError_t launch_matmul_narrow(const MatmulArgs& a, int tokens, int splits, cudaStream_t s) {
  return tokens == 16 ? launch_type<16>(a, splits, s) : tokens == 32 ? launch_type<32>(a, splits, s) : launch_type<64>(a, splits, s);
}

}  // namespace bl
