// The experts of each token, and the lists of rows that they make.
//   chosen   the top_k largest of a token's scores; of equals the lowest index first (a NaN counts as less than -infinity)
//   weights  exp(z_e - max z) over their sum, over the chosen or over all experts
//   offsets  first row of each expert in the list of all (token, choice) pairs ordered by expert, then by token
//   rows     the token of each row of that list;  places: the row of each (token, choice)
// Latency, not bandwidth: the scores of 8191 tokens over 128 experts are 2 MB.  A warp holds a token's scores as keys
// whose unsigned order is theirs (lane l has experts l, l + 32, ..), and picks by warp-wide integer maxima; a 16-bit score and its
// expert share a key, so that one maximum finds both.  A warp's tokens are loaded before the first is looked at.
// The order of the list comes without sorting: each block of kRun tokens notes, per expert, the set of its tokens
// as bits, so a token's rank is a count of lower bits, whatever the order in which warps set them.  With one block that
// is all; with more, each leaves its counts (a byte per expert) and a second kernel adds up those of the
// blocks before its own.  Beyond kDirect blocks, whose counts every block would read, a kernel in between sums them up.
#include "common.cuh"

namespace bl {

namespace {

constexpr int kRun = 64;                       // tokens per block; a count fits a byte
constexpr int kWarps = 32;
constexpr int kThreads = kWarps * 32;
constexpr int kMaxExperts = 512;
constexpr int kDirect = 512;                   // blocks whose counts the placing kernel adds up itself

// Unsigned order of the keys = order of the values; -0 and 0 are equal, NaN is lowest.  Nothing is 0, the key of what is taken or was
// never there.
__device__ __forceinline__ uint32_t key_of(float z) { return (z != z ? 0u : enc_ordered(z + 0.f)) + 1u; }
__device__ __forceinline__ float value_of(uint32_t key) { return dec_ordered(key - 1u); }      // of any but NaN

// Key and expert of a score of 16 bits: equal scores in the order of their experts, lowest first.
template <typename T> __device__ __forceinline__ uint32_t short_key(T v, int e) {
  const float z = in_cast(v) + 0.f;
  const uint32_t b = (uint32_t)*reinterpret_cast<const uint16_t*>(&v);
  const uint32_t order = z != z ? 0u : z == 0.f ? 0x8000u : (b & 0x8000u) ? 0xFFFFu - b : b + 0x8000u;   // +0 is 0x8000, the largest 0xFC00 or less
  return ((order + 1u) << 16) | (uint32_t)(0xFFFF - e);
}

// One warp: first[e] = sum of count[0..e-1].
__device__ __forceinline__ void prefix_sums(int experts, const int* count, int* first) {
  const int lane = threadIdx.x & 31;
  int sum = 0;
  for (int base = 0; base < experts; base += 32) {
    const int e = base + lane, n = e < experts ? count[e] : 0;
    int upto = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xFFFFFFFFu, upto, o);
      if (lane >= o) upto += v;
    }
    if (e < experts) first[e] = sum + upto - n;
    sum += __shfl_sync(0xFFFFFFFFu, upto, 31);
  }
  if (lane == 0) first[experts] = sum;
}

constexpr int kPerWarp = kRun / kWarps;        // tokens

template <typename T, int kPer>                // kPer scores per lane
__global__ void __launch_bounds__(kThreads) route_pick_kernel(RouteArgs a) {
  __shared__ unsigned long long members[kMaxExperts];      // tokens of the run that chose the expert
  __shared__ int count[kMaxExperts], first[kMaxExperts + 1];
  constexpr bool kShort = sizeof(T) == 2;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const bool alone = gridDim.x == 1;
  pdl_launch_dependents();
  for (int e = threadIdx.x; e < a.experts; e += kThreads) members[e] = 0ull;
  __syncthreads();
  pdl_wait();
  const int64_t t0 = (int64_t)blockIdx.x * kRun;
  const T* logits = reinterpret_cast<const T*>(a.logits);
  T raw[kPerWarp][kPer];
  int32_t position[kPerWarp];
#pragma unroll
  for (int n = 0; n < kPerWarp; ++n) {
    const int64_t t = t0 + warp + n * kWarps;
    position[n] = a.positions && t < a.T ? a.positions[t] : 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int e = lane + 32 * i;
      raw[n][i] = t < a.T && e < a.experts ? logits[t * a.ld + e] : T(-INFINITY);
    }
  }
#pragma unroll
  for (int n = 0; n < kPerWarp; ++n) {
    const int local = warp + n * kWarps;
    const int64_t t = t0 + local;
    if (t >= a.T) break;
    const bool padding = position[n] < 0;
    uint32_t key[kPer];
    int expert[kPer];
    bool nan = false;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int e = lane + 32 * i;
      const float z = in_cast(raw[n][i]);
      nan |= z != z;
      expert[i] = e;
      if constexpr (kShort) key[i] = e < a.experts ? short_key(raw[n][i], e) : 0u;
      else key[i] = e < a.experts ? key_of(z) : 0u;
    }
    nan = __any_sync(0xFFFFFFFFu, nan);
    // A lane's scores in order, largest first, equal ones by their experts: a round then looks at the first only.
#pragma unroll
    for (int i = 1; i < kPer; ++i) {
#pragma unroll
      for (int j = i; j > 0; --j) {
        if (key[j] > key[j - 1]) {
          const uint32_t k = key[j]; key[j] = key[j - 1]; key[j - 1] = k;
          if constexpr (!kShort) { const int x = expert[j]; expert[j] = expert[j - 1]; expert[j - 1] = x; }
        }
      }
    }
    // top_k times: the largest key, and of the experts that have it the lowest
    int mine = -1;                             // lane j keeps choice j
    uint32_t mine_key = 0u, top_key = 0u;
    for (int j = 0; j < a.top_k; ++j) {
      const uint32_t best = __reduce_max_sync(0xFFFFFFFFu, key[0]);
      int e;
      bool taken = key[0] == best;
      if constexpr (kShort) {
        e = 0xFFFF - (int)(best & 0xFFFFu);
      } else {
        e = __reduce_min_sync(0xFFFFFFFFu, taken ? expert[0] : INT32_MAX);
        taken = taken && expert[0] == e;
      }
      if (taken) {
#pragma unroll
        for (int i = 0; i + 1 < kPer; ++i) { key[i] = key[i + 1]; if constexpr (!kShort) expert[i] = expert[i + 1]; }
        key[kPer - 1] = 0u;
      }
      if (j == 0) top_key = best;
      if (lane == j) { mine = e; mine_key = best; }
    }
    auto value = [](uint32_t k) {              // of a key; of one that stands for NaN, anything
      if constexpr (kShort) {
        const uint32_t o = (k >> 16) - 1u;
        const uint16_t b = (uint16_t)(o >= 0x8000u ? o - 0x8000u : 0xFFFFu - o);
        return in_cast(*reinterpret_cast<const T*>(&b));
      } else {
        return value_of(k);
      }
    };
    const float top_z = value(top_key);
    float p = lane < a.top_k ? expf(value(mine_key) - top_z) : 0.f, total = p;
    if (!a.normalise) {
      total = 0.f;
#pragma unroll
      for (int i = 0; i < kPer; ++i) if (lane + 32 * i < a.experts) total += expf(in_cast(raw[n][i]) - top_z);
    }
    total = warp_sum(total);
    if (lane < a.top_k) {
      a.chosen[t * a.top_k + lane] = padding ? -1 : mine;
      a.weights[t * a.top_k + lane] = padding ? 0.f : nan ? __uint_as_float(0x7FC00000u) : p / total;
      if (!padding) atomicOr(&members[mine], 1ull << local);
    }
  }
  __syncthreads();
  if (!alone) {
    for (int e = threadIdx.x; e < a.experts; e += kThreads) {
      a.members[(int64_t)blockIdx.x * a.experts + e] = members[e];
      a.counts[(int64_t)blockIdx.x * a.stride + e] = (uint8_t)__popcll(members[e]);
    }
    return;
  }
  // one block: its own prefix sums
  for (int e = threadIdx.x; e < a.experts; e += kThreads) count[e] = __popcll(members[e]);
  __syncthreads();
  if (warp == 0) prefix_sums(a.experts, count, first);
  __syncthreads();
  for (int e = threadIdx.x; e <= a.experts; e += kThreads) a.offsets[e] = first[e];
  for (int c = threadIdx.x; c < (int)a.T * a.top_k; c += kThreads) {
    const int local = c / a.top_k, e = a.chosen[c];
    int place = -1;
    if (e >= 0) {
      place = first[e] + __popcll(members[e] & ((1ull << local) - 1ull));
      a.rows[place] = local;
    }
    a.places[c] = place;
  }
}

// Many blocks: counts summed over all blocks before each, per expert.  One block per expert.
__global__ void __launch_bounds__(256) route_sum_kernel(RouteArgs a, int runs) {
  __shared__ int part[8];
  pdl_launch_dependents();
  pdl_wait();
  const int e = blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int before = 0;
  for (int base = 0; base < runs; base += 256) {
    const int r = base + threadIdx.x;
    const int n = r < runs ? a.counts[(int64_t)r * a.stride + e] : 0;
    int upto = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xFFFFFFFFu, upto, o);
      if (lane >= o) upto += v;
    }
    if (lane == 31) part[warp] = upto;
    __syncthreads();
    int lower = 0, all = 0;
#pragma unroll
    for (int w = 0; w < 8; ++w) { if (w < warp) lower += part[w]; all += part[w]; }
    if (r < runs) a.sums[(int64_t)r * a.experts + e] = before + lower + upto - n;
    before += all;
    __syncthreads();
  }
  if (threadIdx.x == 0) a.sums[(int64_t)runs * a.experts + e] = before;
}

// Rows and places of a run, and the offsets.
template <bool kSummed>
__global__ void __launch_bounds__(kThreads) route_place_kernel(RouteArgs a, int runs) {
  __shared__ int total[kMaxExperts], before[kMaxExperts];
  __shared__ int first[kMaxExperts + 1];
  __shared__ unsigned long long members[kMaxExperts];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  pdl_launch_dependents();
  for (int e = threadIdx.x; e < a.experts; e += kThreads) { total[e] = 0; before[e] = 0; }
  __syncthreads();
  pdl_wait();
  // What the end needs is asked for first.
  const int64_t t0 = (int64_t)blockIdx.x * kRun;
  const int here = (int)min((int64_t)kRun, a.T - t0) * a.top_k;      // choices of the run, at most two for each thread
  const int32_t* chosen = a.chosen + t0 * a.top_k;
  const int e0 = threadIdx.x < here ? chosen[threadIdx.x] : -1, e1 = threadIdx.x + kThreads < here ? chosen[threadIdx.x + kThreads] : -1;
  for (int e = threadIdx.x; e < a.experts; e += kThreads) members[e] = a.members[(int64_t)blockIdx.x * a.experts + e];
  if (kSummed) {
    for (int e = threadIdx.x; e < a.experts; e += kThreads) {
      total[e] = a.sums[(int64_t)runs * a.experts + e];
      before[e] = a.sums[(int64_t)blockIdx.x * a.experts + e];
    }
  } else {
    // four experts a thread (the rows of counts are padded to words), the runs shared out over the warps; sums of up to 16 runs of 64
    // tokens, two in a word
    const int words = a.stride / 4;
    for (int w0 = 0; w0 < words; w0 += 32) {
      const int w = w0 + lane;
      uint32_t all[2] = {0u, 0u}, low[2] = {0u, 0u};
      if (w < words) {
#pragma unroll 4
        for (int r = warp; r < runs; r += kWarps) {
          const uint32_t c = *reinterpret_cast<const uint32_t*>(a.counts + (int64_t)r * a.stride + 4 * w);
          const uint32_t even = c & 0x00FF00FFu, odd = (c >> 8) & 0x00FF00FFu;
          all[0] += even; all[1] += odd;
          if (r < (int)blockIdx.x) { low[0] += even; low[1] += odd; }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {                  // whole numbers: any order
          if (4 * w + i >= a.experts) break;
          atomicAdd(&total[4 * w + i], (int)(all[i & 1] >> (16 * (i >> 1)) & 0xFFFFu));
          atomicAdd(&before[4 * w + i], (int)(low[i & 1] >> (16 * (i >> 1)) & 0xFFFFu));
        }
      }
    }
  }
  __syncthreads();
  if (warp == 0) prefix_sums(a.experts, total, first);
  __syncthreads();
  if (blockIdx.x == 0)
    for (int e = threadIdx.x; e <= a.experts; e += kThreads) a.offsets[e] = first[e];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int c = threadIdx.x + k * kThreads, e = k ? e1 : e0;
    if (c >= here) break;
    int place = -1;
    if (e >= 0) {
      const int local = c / a.top_k;
      place = first[e] + before[e] + __popcll(members[e] & ((1ull << local) - 1ull));
      a.rows[place] = (int)(t0 + local);
    }
    a.places[t0 * a.top_k + c] = place;
  }
}

// Many blocks: one per SM.  They need few registers, and two on an SM while another has none take as long as two (8191 tokens over 128
// experts 13.1 us, so 9.1): each asks for more than half of the shared memory.
constexpr size_t kAlone = 120 * 1024;

template <typename T, int kPer>
cudaError_t pick_per(const RouteArgs& a, unsigned runs, cudaStream_t s) {
  const auto kern = route_pick_kernel<T, kPer>;
  if (runs == 1) return launch_pdl(kern, runs, kThreads, 0, s, a);
  static std::atomic<uint64_t> ready{0};                     // devices on which the kernel's shared memory limit is set
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev > 63 || !(ready.load(std::memory_order_acquire) >> dev & 1)) {
    if ((e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kAlone)) != cudaSuccess) return e;
    if (dev <= 63) ready.fetch_or(1ull << dev, std::memory_order_acq_rel);
  }
  return launch_pdl(kern, runs, kThreads, kAlone, s, a);
}

template <typename T>
cudaError_t pick(const RouteArgs& a, unsigned runs, cudaStream_t s) {
  if (a.experts <= 32) return pick_per<T, 1>(a, runs, s);
  if (a.experts <= 64) return pick_per<T, 2>(a, runs, s);
  if (a.experts <= 128) return pick_per<T, 4>(a, runs, s);
  if (a.experts <= 256) return pick_per<T, 8>(a, runs, s);
  return pick_per<T, 16>(a, runs, s);
}

size_t round16(size_t v) { return (v + 15) & ~size_t(15); }

struct Carve { size_t members, counts, sums, total; };
Carve carve(int64_t T, int experts) {
  Carve c{0, 0, 0, 0};
  const size_t runs = (size_t)((T + kRun - 1) / kRun);
  if (runs <= 1) return c;
  const size_t stride = (size_t)((experts + 3) / 4 * 4);
  c.counts = round16(runs * (size_t)experts * 8);
  c.sums = c.counts + round16(runs * stride);
  c.total = c.sums + (runs > kDirect ? (runs + 1) * (size_t)experts * 4 : 0);
  return c;
}

}  // namespace

size_t route_topk_ws_bytes(int64_t T, int experts) { return carve(T, experts).total; }

cudaError_t launch_route_topk(RouteArgs a, void* ws, cudaStream_t s) {
  const Carve c = carve(a.T, a.experts);
  const unsigned runs = a.T > 0 ? (unsigned)((a.T + kRun - 1) / kRun) : 1u;
  a.stride = (a.experts + 3) / 4 * 4;
  a.members = reinterpret_cast<unsigned long long*>(ws);
  a.counts = reinterpret_cast<uint8_t*>(ws) + c.counts;
  a.sums = reinterpret_cast<int32_t*>(reinterpret_cast<uint8_t*>(ws) + c.sums);
  cudaError_t e = a.dt == BL_F32 ? pick<float>(a, runs, s) : a.dt == BL_F16 ? pick<__half>(a, runs, s) : pick<__nv_bfloat16>(a, runs, s);
  if (e != cudaSuccess || runs == 1) return e;
  if (runs <= kDirect) return launch_pdl(route_place_kernel<false>, runs, kThreads, 0, s, a, (int)runs);
  if ((e = launch_pdl(route_sum_kernel, (unsigned)a.experts, 256, 0, s, a, (int)runs)) != cudaSuccess) return e;
  return launch_pdl(route_place_kernel<true>, runs, kThreads, 0, s, a, (int)runs);
}

}  // namespace bl
