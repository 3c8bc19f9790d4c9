// Attention of the last n_q tokens of each sequence over the 4-bit paged cache:
//   s_jr = scale . q_r . (eta_j + step_j c_j),  o_r = sum_j p_jr (eta'_j + step'_j c'_j) / sum_j p_jr,  p = e^(s - max).
// Bound by reading the cache (kDim + 8 bytes per token and head); everything below serves to keep up with that.
//
// Products.  Codes are never turned into values: with the step and eta of a token outside the sums,
//   s_jr = scale (step_j (q_r . c_j) + eta_j sum q_r),   o_r = sum_j (p_jr step'_j) c'_j + sum_j p_jr eta'_j,
// both products are exact integers 0..15 times 16-bit numbers on the tensor cores (mma m16n8k16, fp32 sums).
// A nibble becomes an fp16 operand by a mask alone: bits 0-3 of a half are the subnormal c . 2^-24, bits 4-7
// are c . 2^-20 (undone in the query operand, or in the output); one shift serves the upper two nibbles.  So 8 codes
// cost 5 instructions.  The tokens are the rows (16) of both products and the query rows (queries x heads of one
// key/value head) the columns (8), so with up to 8 query rows no tensor work is idle on a padded dimension of 16;
// the probabilities pass from the first product's layout to the second's by an 8x8 transposition in registers.
// The cache's orders are such that a lane's operands of 8 tokens are 16 contiguous bytes.
//
// Precision.  The query operand is the query times a power of two that puts the row's largest value at 2^13 (exact
// unless a value is 2^-24 of the largest and more below it).  p . step' is rounded to fp16 after scaling by a running power of two (2^13 / largest
// step' so far), so its range is 2^-37 of the largest.  The codes' mean is taken out of its rounding error: with
// u = fp16(p step'), o = sum u (c' - 7.5) + sum p (eta' + 7.5 step'), where sum u comes from one more product
// with a tile of ones.  Everything else
// (scores, statistics, eta sums, accumulators) is fp32.  Against products in fp32 throughout the two roundings raise the error from
// 2.1e-4 to 3.0e-4 of the result (fp16, 32 x 8192 tokens) and from 1.6e-3 to 1.8e-3 (bf16, 2 x 150001), most of it the output's own.
//
// Work.  The visible tokens of all sequences, in chunks of 64, times key/value heads (times blocks of query rows)
// form one list that is cut into equal parts, one per warp: ragged batches and single long sequences balance
// alike.  A warp runs on its own: its chunks stream into its part of shared memory by bulk copies, one or two ahead
// (104 or 139 KB in flight per SM), with no barrier between warps.  The wait for a chunk is bounded; one that runs out is
// reported in the warp's status word, and the rows that the warp still had to work on become NaN.  A warp that owns
// all chunks of a head writes the output; else its unnormalised sums go to the workspace, two slots per warp, and a second
// kernel joins them in list order.
// Few and short lists go to clusters of CTAs instead, one per list (a sequence, key/value head and block of rows), which
// join their parts through each other's shared memory: one kernel (launch_dim gives the rule).
#include <algorithm>
#include <type_traits>

#include "kv4.cuh"
#include "tc_common.cuh"

namespace bl {

namespace {

using namespace kv4;

constexpr int kChunk = 64;                 // tokens per work item
constexpr int kMostWarps = 12;             // per CTA, one CTA per SM
constexpr int kMaxSms = 160;
constexpr int kMostClusterLog2 = 3, kMostCluster = 1 << kMostClusterLog2;   // CTAs of a cluster
constexpr int kCtaRows = 4;                // rows of the result per SM up to which the join has a CTA for each
constexpr int kClusterChunks = 4;          // chunks per warp up to which a cluster takes a list
constexpr size_t kStatusBytes = 7936;      // the status words lie at the start of the workspace
static_assert((1 + kMaxSms * kMostWarps) * 4 <= kStatusBytes && kMaxSms * kMostWarps <= (int)kMostStatusWords, "more warps than status words");

struct Plan {                              // how the list is laid out; made on the host, the same for both kernels
  int group, rows, rows_per_block, blocks; // query heads per key/value head; query rows; rows per block; blocks
  int heads_blocks;                        // key/value heads x blocks
  int page_log2, parts;                    // log2 page_size; parts of the list (warps)
  int cluster_log2;                        // log2 CTAs of a cluster, where each works on a list of its own
  uint32_t parts_magic;                    // floor(2^32 / parts) + 1
};
inline Plan make_plan(int n_q, int heads, int kv_heads, int page_size, int parts, int cluster_log2 = 0) {
  Plan p;
  p.cluster_log2 = cluster_log2;
  p.group = heads / kv_heads;
  p.rows = n_q * p.group;
  p.rows_per_block = p.rows <= 8 ? p.rows : 16;
  p.blocks = (p.rows + p.rows_per_block - 1) / p.rows_per_block;
  p.heads_blocks = kv_heads * p.blocks;
  p.page_log2 = page_size == 16 ? 4 : page_size == 32 ? 5 : 6;
  p.parts = parts;
  p.parts_magic = (uint32_t)((1ull << 32) / (unsigned)parts) + 1;
  return p;
}

// The chunks of one sequence that hold a visible token: those of the sinks, then those from the window's begin on.
struct Seq {
  int len, lo;                             // tokens; first token inside the first query's window
  int sink_chunks, first_main, chunks;
  __device__ __forceinline__ int start(int c) const { return (c < sink_chunks ? c : first_main + c - sink_chunks) * kChunk; }
};
__device__ __forceinline__ Seq make_seq(const Kv4AttnArgs& a, int b) {
  Seq s;
  s.len = (int)min((int64_t)max(a.lens[b], 0), a.max_pages * a.cache.page_size);
  s.lo = a.window > 0 ? max(0, max(0, s.len - a.n_q) - a.window + 1) : 0;
  s.first_main = s.lo / kChunk;
  s.sink_chunks = min((int)(((int64_t)min(a.sinks, s.lo) + kChunk - 1) / kChunk), s.first_main);
  s.chunks = s.len > 0 ? s.sink_chunks + (s.len + kChunk - 1) / kChunk - s.first_main : 0;
  return s;
}

// Where the sequences' chunks lie in one row of numbers (by a whole warp).  Up to 32 sequences: found out once, each lane
// keeping one; more: added up again when asked.
struct Spread {
  int mine, upto;                          // chunks of sequence `lane`, and of those up to it
  int64_t all;                             // chunks of all sequences
  __device__ __forceinline__ explicit Spread(const Kv4AttnArgs& a) {
    const int lane = threadIdx.x & 31;
    all = 0;
    for (int base = 0; base < a.batch; base += 32) {
      scan(base + lane < a.batch ? make_seq(a, base + lane).chunks : 0);
      all += __shfl_sync(0xFFFFFFFFu, upto, 31);
    }
  }
  __device__ __forceinline__ void scan(int n) {
    const int lane = threadIdx.x & 31;
    mine = upto = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int up = __shfl_up_sync(0xFFFFFFFFu, upto, o);
      if (lane >= o) upto += up;
    }
  }
  // The sequence that item `at` of the list falls into, and the item's place among that sequence's.
  __device__ __forceinline__ int find(const Kv4AttnArgs& a, int heads_blocks, int64_t at, int64_t& rest) {
    const int lane = threadIdx.x & 31;
    int64_t before = 0;
    for (int base = 0; base < a.batch; base += 32) {
      if (a.batch > 32) scan(base + lane < a.batch ? make_seq(a, base + lane).chunks : 0);
      const unsigned past = __ballot_sync(0xFFFFFFFFu, (before + upto) * heads_blocks > at);
      if (past) {
        const int f = __ffs(past) - 1;
        rest = at - (before + __shfl_sync(0xFFFFFFFFu, upto - mine, f)) * heads_blocks;
        return base + f;
      }
      before += __shfl_sync(0xFFFFFFFFu, upto, 31);
    }
    rest = 0;
    return a.batch;
  }
};

// Workspace: the status words (one per warp), the parts (two slots per warp), then two numbers per sequence, head and block of rows.
__host__ __device__ inline int64_t slot_floats(const Plan& plan, int head_dim) { return (int64_t)plan.rows_per_block * (head_dim + 4); }
__device__ __forceinline__ float* slots_of(const Kv4AttnArgs& a) { return reinterpret_cast<float*>(reinterpret_cast<char*>(a.ws) + kStatusBytes); }
__device__ __forceinline__ int* ends_of(const Kv4AttnArgs& a, const Plan& plan) {
  return reinterpret_cast<int*>(slots_of(a) + 2 * plan.parts * slot_floats(plan, a.cache.head_dim));
}

// The warps of the launch in one row of numbers (those of a CTA far apart: short lists spread over the SMs), and a warp's status word.
__device__ __forceinline__ int warp_number() { return (int)((threadIdx.x >> 5) * gridDim.x + blockIdx.x); }
__device__ __forceinline__ void set_status(void* ws, uint32_t status) { reinterpret_cast<volatile uint32_t*>(ws)[1 + warp_number()] = status; }

// a / b for a >= 0, b > 0: the 32-bit division (a fifth of the instructions) where it serves.
__device__ __forceinline__ int64_t divide(int64_t a, int64_t b) {
  return ((a | b) >> 32) == 0 ? (int64_t)((uint32_t)a / (uint32_t)b) : a / b;
}
// The cut of a list of items into parts: part w starts at begin(w).
struct Cut {
  int64_t each; int more;                  // items of a part; the first `more` parts have one more
  __device__ __forceinline__ Cut(int64_t total, const Plan& plan) {
    if (total >> 31) {
      each = total / plan.parts;
    } else {                               // n / parts is at most half a unit below n magic / 2^32 for n < 2^31
      const uint32_t n = (uint32_t)total, q = __umulhi(n, plan.parts_magic);
      each = q * (uint32_t)plan.parts > n ? q - 1 : q;
    }
    more = (int)(total - each * plan.parts);
  }
  __device__ __forceinline__ int64_t begin(int w) const { return each * w + min(w, more); }
};

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
// kBytes contiguous bytes by the copy engine, counted on a barrier (both addresses and the size are multiples of 16).
__device__ __forceinline__ void copy_bulk(uint32_t dst, const void* src, int bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
// Barrier of a cluster's threads; a number in the shared memory of its CTA `rank`, at p in one's own.
__device__ __forceinline__ void cluster_meet() {
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ float2 peer_float2(const float* p, int rank) {
  uint32_t addr;
  float2 v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(addr) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
  asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(addr) : "memory");
  return v;
}
// Whether a part with this maximum and sum of a row holds nothing that the row sees.  The maximum alone does not say: fmaxf passes
// NaN over, so a row of scores that are NaN, or all -infinity, has a maximum of -infinity too, and a sum that is NaN.
__device__ __forceinline__ bool sees_nothing(float top, float sum) { return top == -INFINITY && sum == 0.f; }
__device__ __forceinline__ uint32_t half2_bits(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// 2^e as a float, e in -126..127
__device__ __forceinline__ float pow2i(int e) { return __int_as_float((e + 127) << 23); }
__device__ __forceinline__ int exponent(float x) { return ((__float_as_int(x) >> 23) & 255) - 127; }

// Larger of two (step, eta) words, each half for itself; a NaN gives way.
template <typename T> __device__ __forceinline__ uint32_t max_pairs(uint32_t a, uint32_t b);
template <> __device__ __forceinline__ uint32_t max_pairs<__half>(uint32_t a, uint32_t b) {
  const __half2 m = __hmax2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
  return *reinterpret_cast<const uint32_t*>(&m);
}
template <> __device__ __forceinline__ uint32_t max_pairs<__nv_bfloat16>(uint32_t a, uint32_t b) {
  const __nv_bfloat162 m = __hmax2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
  return *reinterpret_cast<const uint32_t*>(&m);
}

template <typename T> __device__ __forceinline__ float2 pair_floats(uint32_t w) { return scale_floats<T>(w); }
template <typename T> __device__ __forceinline__ uint32_t pair_bits(float lo, float hi);
template <> __device__ __forceinline__ uint32_t pair_bits<__half>(float lo, float hi) { return half2_bits(lo, hi); }
template <> __device__ __forceinline__ uint32_t pair_bits<__nv_bfloat16>(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// Walks the items of a warp's part of the list.
struct Walk {
  Seq s;
  int b, hk, blk, c;                       // sequence, key/value head, block of query rows, chunk
  __device__ __forceinline__ void next(const Kv4AttnArgs& a, const Plan& plan) {
    if (++c < s.chunks) return;
    c = 0;
    if (++blk < plan.blocks) return;
    blk = 0;
    if (++hk < a.cache.kv_heads) return;
    hk = 0;
    do { ++b; } while (b < a.batch && (s = make_seq(a, b)).chunks == 0);
  }
};

// Words of shared memory read as operands: 4 words for kDim 128, 2 for kDim 64.
template <int kWords> __device__ __forceinline__ void load_words(const char* p, uint32_t (&w)[kWords]);
template <> __device__ __forceinline__ void load_words<4>(const char* p, uint32_t (&w)[4]) {
  const uint4 r = *reinterpret_cast<const uint4*>(p);
  w[0] = r.x; w[1] = r.y; w[2] = r.z; w[3] = r.w;
}
template <> __device__ __forceinline__ void load_words<2>(const char* p, uint32_t (&w)[2]) {
  const uint2 r = *reinterpret_cast<const uint2*>(p);
  w[0] = r.x; w[1] = r.y;
}

// The two numbers by which the join finds a row block's parts: the slot of the first chunk's, the warp of the last chunk's.
__device__ __forceinline__ int* ends_at(const Kv4AttnArgs& a, const Plan& plan, int b, int hk, int blk) {
  return ends_of(a, plan) + 2 * (((int64_t)b * a.cache.kv_heads + hk) * plan.blocks + blk);
}

// The warp's copies did not come: the rows of its items from `item` on (later: an item before it ended a segment; from_start: the
// segment that it goes on with began with its list's first chunk) become NaN, a part's sum where they are not the warp's alone,
// which goes through every join.  Out of line, with a walk of its own: the loop over the chunks has no register to spare for it.
template <typename T, int kDim>
__device__ __noinline__ void lose_items(Kv4AttnArgs a, Plan plan, int item, bool later, bool from_start, bool fresh) {
  const int lane = threadIdx.x & 31, w = warp_number();
  const float nan = __int_as_float(0x7FC00000);
  Spread spread(a);
  const Cut cut(spread.all * plan.heads_blocks, plan);
  const int64_t end = cut.begin(w + 1);
  int64_t at = cut.begin(w) + item, rest;
  Walk x;
  x.b = spread.find(a, plan.heads_blocks, at, rest);
  x.s = make_seq(a, x.b);
  const int hb = (int)(rest / x.s.chunks);
  x.c = (int)(rest - (int64_t)hb * x.s.chunks);
  x.hk = hb / plan.blocks;
  x.blk = hb - x.hk * plan.blocks;
  while (at < end) {                                   // a segment each time: all that is left of a list, or of the warp's items
    if (fresh) from_start = x.c == 0;
    const int n = (int)min((int64_t)(x.s.chunks - x.c), end - at);
    const bool last = x.c + n == x.s.chunks;
    float* slot = slots_of(a) + (2 * w + later) * slot_floats(plan, kDim);
    if (lane == 0) {
      int* where = ends_at(a, plan, x.b, x.hk, x.blk);
      if (from_start) where[0] = 2 * w + later;
      if (last) where[1] = w;
    }
    for (int rr = 0; rr < min(plan.rows_per_block, plan.rows - x.blk * plan.rows_per_block); ++rr) {
      const int r = x.blk * plan.rows_per_block + rr, i_q = r / plan.group;
      T* out = reinterpret_cast<T*>(a.o) + ((int64_t)x.b * a.n_q + i_q) * a.ld_o + (int64_t)(x.hk * plan.group + r - i_q * plan.group) * kDim;
      if (from_start && last) {
        for (int d = lane; d < kDim; d += 32) out[d] = out_cast<T>(nan);
      } else if (lane == 0) {
        *reinterpret_cast<float2*>(slot + rr * (kDim + 4) + kDim) = make_float2(-INFINITY, nan);
      }
    }
    later = fresh = true;
    at += n;
    x.c += n - 1;
    if (at < end) x.next(a, plan);
  }
}

// What a chunk in flight is, written beside its bytes when its copies are issued.
struct __align__(16) Item {
  int t0, len, b, hk;                      // first token, tokens of its sequence, sequence, key/value head
  int rows0, there, first, last;           // first query row; which runs of tokens are there (bit per page); first, last chunk of its list
};

// kNT: tiles of 8 query rows; kWarps per CTA, each with kStages chunks in shared memory; kCluster: a cluster per list.
template <typename T, int kDim, int kNT, int kWarps, int kStages, bool kCluster>
__global__ void __launch_bounds__(kWarps * 32, 1) attention_kv4_kernel(Kv4AttnArgs a, Plan plan, uint32_t polls) {
  constexpr int kWords = kDim / 32;        // words of codes per lane and 8 tokens
  constexpr int kTiles = kChunk / 16;
  constexpr int kStageBytes = kChunk * (kDim + 8);
  constexpr uint32_t kLo = 0x000F000Fu, kHi = 0x00F000F0u, kOnes = 0x3C003C00u;
  extern __shared__ __align__(16) char smem[];
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, qd = lane & 3;
  const int w = warp_number();
  const int ps = a.cache.page_size, pl = plan.page_log2, block_bytes = Block<kDim>::bytes(ps), subs = kChunk >> pl;
  char* ring = smem + warp * (kStages * kStageBytes);
  const uint32_t ring_addr = (uint32_t)__cvta_generic_to_shared(ring);
  Item* items_of = reinterpret_cast<Item*>(smem + kWarps * kStages * kStageBytes) + warp * kStages;
  const uint32_t bar_addr = (uint32_t)__cvta_generic_to_shared(smem + kWarps * kStages * (kStageBytes + sizeof(Item))) + warp * kStages * 8;
  if (lane == 0) {
    for (int i = 0; i < kStages; ++i) tc::mbar_init(bar_addr + 8 * i, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncwarp();

  pdl_wait();
  if (blockIdx.x == 0 && threadIdx.x == 0) *reinterpret_cast<uint32_t*>(a.ws) = kStatusPerWarp + gridDim.x * kWarps;
  if (lane == 0) set_status(a.ws, 0);
  // ---- loads: the page numbers of a chunk are fetched one chunk before its copies are issued
  Walk ahead;
  int items;
  const int rank = blockIdx.x & ((1 << plan.cluster_log2) - 1);
  if (kCluster) {                                      // the chunks of the cluster's list, cut for its warps
    const int unit = blockIdx.x >> plan.cluster_log2, part = (warp << plan.cluster_log2) + rank;
    ahead.b = unit / plan.heads_blocks;
    const int hb = unit - ahead.b * plan.heads_blocks;
    ahead.s = make_seq(a, ahead.b);
    ahead.hk = hb / plan.blocks;
    ahead.blk = hb - ahead.hk * plan.blocks;
    ahead.c = (int)((uint32_t)(ahead.s.chunks * part) / (uint32_t)plan.parts);
    items = (int)((uint32_t)(ahead.s.chunks * (part + 1)) / (uint32_t)plan.parts) - ahead.c;
  } else {
    Spread spread(a);
    const Cut cut(spread.all * plan.heads_blocks, plan);
    const int64_t begin = cut.begin(w);
    items = (int)(cut.begin(w + 1) - begin);
    if (items == 0) return;
    int64_t rest;
    ahead.b = spread.find(a, plan.heads_blocks, begin, rest);
    ahead.s = make_seq(a, ahead.b);
    const int hb = (int)divide(rest, ahead.s.chunks);
    ahead.c = (int)(rest - (int64_t)hb * ahead.s.chunks);
    ahead.hk = plan.blocks == 1 ? hb : hb / plan.blocks;
    ahead.blk = hb - ahead.hk * plan.blocks;
  }
  auto page_of = [&](const Walk& x) -> int {           // lane i: the page of the chunk's i-th run of tokens; -1: nothing visible, or no page
    if (lane >= subs) return -1;
    const int t = x.s.start(x.c) + lane * ps;
    if (t >= x.s.len || (t + ps <= x.s.lo && t >= a.sinks)) return -1;
    const int id = a.table[(int64_t)x.b * a.max_pages + (t >> pl)];
    return id >= 0 && id < a.cache.num_pages ? id : -1;
  };
  int issued = 0;
  int ids = items > 0 ? page_of(ahead) : -1;
  auto issue = [&]() {
    if (issued < items) {
      const int slot = issued % kStages;
      const uint32_t dst = ring_addr + slot * kStageBytes;
      const int there = (int)__ballot_sync(0xFFFFFFFFu, ids >= 0);
      if (lane == 0) {
        Item x;
        x.t0 = ahead.s.start(ahead.c); x.len = ahead.s.len; x.b = ahead.b; x.hk = ahead.hk;
        x.rows0 = ahead.blk * plan.rows_per_block; x.there = there; x.first = ahead.c == 0; x.last = ahead.c + 1 == ahead.s.chunks;
        items_of[slot] = x;
      }
      if (lane == 0) tc::mbar_arrive_expect_tx(bar_addr + 8 * slot, __popc(there) * block_bytes);
      __syncwarp();
      if (ids >= 0)                                    // lane i copies the i-th page's block
        copy_bulk(dst + lane * block_bytes, reinterpret_cast<const char*>(a.cache.pages) + ((int64_t)ids * a.cache.kv_heads + ahead.hk) * block_bytes,
                  block_bytes, bar_addr + 8 * slot);
      if (issued + 1 < items) {
        if (kCluster) ++ahead.c; else ahead.next(a, plan);
        ids = page_of(ahead);
      }
    }
    ++issued;
  };
#pragma unroll
  for (int i = 0; i < kStages - 1; ++i) issue();

  // where tile i (16 tokens) of a stage has its key codes and its key (step, eta) pairs; those of the values follow
  // v_off and 4 ps bytes later
  int code_at[kTiles], scale_at[kTiles];
#pragma unroll
  for (int i = 0; i < kTiles; ++i) {
    const int j0 = (i * 16) & (ps - 1), base = (i * 16 >> pl) * block_bytes;
    code_at[i] = base + j0 * (kDim / 2) + lane * (kWords * 4);
    scale_at[i] = base + Block<kDim>::k_scale(ps) + 4 * (j0 + g);
  }
  const int v_off = Block<kDim>::v_codes(ps);

  // ---- state of the segment (one sequence, head and block of rows) being worked on
  uint32_t qf[kNT][kWords][4];                         // query operand: per word of codes the pairs (0,4), (1,5)/16, (2,6), (3,7)/16
  float f[kNT][2], qsum[kNT][2];                       // per column: scale of the raw score, scaled sum of the query
  float acc[kNT][2 * kWords][4];
  float m[kNT][2], l[kNT][2], esum[kNT][2];
  float usum[kNT][4];                                  // sums of the rounded p . step' (every row of the tile alike)
  int vexp[kNT][2];                                    // 2^vexp: running size of the value steps that the row has seen
  int back_first = 0, back_last = 0;                   // positions of the block's first and last query, back from the sequence's end
  bool from_start = false, later = false;              // the segment began with its list's first chunk; it is not the warp's first

  auto begin_segment = [&](const Item& it) {
    from_start = it.first;
    back_first = a.n_q - it.rows0 / plan.group;
    back_last = a.n_q - (min(it.rows0 + plan.rows_per_block, plan.rows) - 1) / plan.group;
    const float sl = a.scale * 1.4426950408889634f;
#pragma unroll
    for (int nt = 0; nt < kNT; ++nt) {
      const int r = it.rows0 + nt * 8 + g, i_q = r / plan.group;
      const bool on = r < plan.rows;
      const T* q = reinterpret_cast<const T*>(a.q) + ((int64_t)it.b * a.n_q + i_q) * a.ld_q +
                   (int64_t)(it.hk * plan.group + r - i_q * plan.group) * kDim + qd * (kDim / 4);
      float v[kWords][8], top = 0.f, sum = 0.f;
#pragma unroll
      for (int i = 0; i < kWords; ++i) {
        const uint4 x = on ? *reinterpret_cast<const uint4*>(q + 8 * i) : make_uint4(0, 0, 0, 0);
        const uint32_t xs[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 y = pair_floats<T>(xs[j]);
          v[i][2 * j] = y.x; v[i][2 * j + 1] = y.y;
          top = fmaxf(top, fmaxf(fabsf(y.x), fabsf(y.y)));
          sum += y.x + y.y;
        }
      }
      top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1)); top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
      sum += __shfl_xor_sync(0xFFFFFFFFu, sum, 1); sum += __shfl_xor_sync(0xFFFFFFFFu, sum, 2);
      const int e = min(13 - exponent(top), 100);      // the largest value goes to 2^13 (all zero: any scale)
      const float up = pow2i(max(e, -114));
#pragma unroll
      for (int i = 0; i < kWords; ++i) {
        qf[nt][i][0] = half2_bits(v[i][0] * up, v[i][4] * up);
        qf[nt][i][1] = half2_bits(v[i][1] * up * 0.0625f, v[i][5] * up * 0.0625f);
        qf[nt][i][2] = half2_bits(v[i][2] * up, v[i][6] * up);
        qf[nt][i][3] = half2_bits(v[i][3] * up * 0.0625f, v[i][7] * up * 0.0625f);
      }
      const float fr = sl * pow2i(-max(e, -114)) * 16777216.f, sr = sum * sl;   // (2^(24 - e) itself may pass 2^127)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        f[nt][j] = __shfl_sync(0xFFFFFFFFu, fr, 4 * (2 * qd + j));
        qsum[nt][j] = __shfl_sync(0xFFFFFFFFu, sr, 4 * (2 * qd + j));
        m[nt][j] = -INFINITY;
        l[nt][j] = esum[nt][j] = 0.f;
        vexp[nt][j] = -1000;
      }
      usum[nt][0] = usum[nt][1] = usum[nt][2] = usum[nt][3] = 0.f;
#pragma unroll
      for (int t = 0; t < 2 * kWords; ++t) acc[nt][t][0] = acc[nt][t][1] = acc[nt][t][2] = acc[nt][t][3] = 0.f;
    }
  };

  // One chunk; kMask: some query of the block does not see some token of it.
  auto chunk = [&](const char* stage, const Item& it, auto masked) {
    constexpr bool kMask = decltype(masked)::value;
    // ---- scores: tile i, rows g and g + 8 (tokens), columns 2 qd and 2 qd + 1 of each 8 query rows
    float s[kTiles][kNT][4];
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
      uint32_t x[kWords], y[kWords];
      load_words<kWords>(stage + code_at[i], x);
      load_words<kWords>(stage + code_at[i] + 4 * kDim, y);
#pragma unroll
      for (int nt = 0; nt < kNT; ++nt) s[i][nt][0] = s[i][nt][1] = s[i][nt][2] = s[i][nt][3] = 0.f;
#pragma unroll
      for (int k = 0; k < kWords; ++k) {
        const uint32_t xs = x[k] >> 8, ys = y[k] >> 8;
#pragma unroll
        for (int nt = 0; nt < kNT; ++nt) {
          mma16816(s[i][nt], x[k] & kLo, y[k] & kLo, x[k] & kHi, y[k] & kHi, qf[nt][k][0], qf[nt][k][1]);
          mma16816(s[i][nt], xs & kLo, ys & kLo, xs & kHi, ys & kHi, qf[nt][k][2], qf[nt][k][3]);
        }
      }
    }
    // scaled, their largest per query row, and the largest value step
    float mx[kNT][2];
    uint32_t vs[kTiles][2], vmax[kMask ? kNT : 1][kMask ? 2 : 1] = {};   // largest value step: of all, or of those that a query sees
    uint32_t seen = 0;                                 // 4 bits per tile and 8 query rows, as s[i][nt]
    int pos_of[kNT][2];
    if (kMask) {
#pragma unroll
      for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
        for (int j = 0; j < 2; ++j) pos_of[nt][j] = it.len - a.n_q + min(it.rows0 + nt * 8 + 2 * qd + j, plan.rows - 1) / plan.group;
    }
#pragma unroll
    for (int nt = 0; nt < kNT; ++nt) { mx[nt][0] = m[nt][0]; mx[nt][1] = m[nt][1]; }
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
      const char* se = stage + scale_at[i];
      const float2 k0 = scale_floats<T>(*reinterpret_cast<const uint32_t*>(se));
      const float2 k1 = scale_floats<T>(*reinterpret_cast<const uint32_t*>(se + 32));
      vs[i][0] = *reinterpret_cast<const uint32_t*>(se + 4 * ps);
      vs[i][1] = *reinterpret_cast<const uint32_t*>(se + 4 * ps + 32);
#pragma unroll
      for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 kk = e < 2 ? k0 : k1;
          s[i][nt][e] = fmaf(s[i][nt][e] * f[nt][e & 1], kk.x, kk.y * qsum[nt][e & 1]);
          if (kMask) {
            const int t = it.t0 + i * 16 + g + (e >> 1) * 8, pos = pos_of[nt][e & 1];
            const bool v = t <= pos && ((it.there >> (i * 16 >> pl)) & 1) && (a.window == 0 || pos - t < a.window || t < a.sinks);
            if (v) {
              seen |= 1u << ((i * kNT + nt) * 4 + e);
              vmax[kMask ? nt : 0][kMask ? e & 1 : 0] = max_pairs<T>(vmax[kMask ? nt : 0][kMask ? e & 1 : 0], vs[i][e >> 1]);
            } else {
              s[i][nt][e] = -INFINITY;
            }
          }
          mx[nt][e & 1] = fmaxf(mx[nt][e & 1], s[i][nt][e]);
        }
      if (!kMask) vmax[0][0] = max_pairs<T>(vmax[0][0], max_pairs<T>(vs[i][0], vs[i][1]));
    }
#pragma unroll
    for (int o = 4; o < 32; o <<= 1) {
#pragma unroll
      for (int nt = 0; nt < kNT; ++nt) {
        mx[nt][0] = fmaxf(mx[nt][0], __shfl_xor_sync(0xFFFFFFFFu, mx[nt][0], o));
        mx[nt][1] = fmaxf(mx[nt][1], __shfl_xor_sync(0xFFFFFFFFu, mx[nt][1], o));
      }
#pragma unroll
      for (int nt = 0; nt < (kMask ? kNT : 1); ++nt)
#pragma unroll
        for (int j = 0; j < (kMask ? 2 : 1); ++j) vmax[nt][j] = max_pairs<T>(vmax[nt][j], __shfl_xor_sync(0xFFFFFFFFu, vmax[nt][j], o));
    }
    int ve[kNT][2];
    bool moved = false;
#pragma unroll
    for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        ve[nt][j] = max(vexp[nt][j], max(exponent(scale_floats<T>(vmax[kMask ? nt : 0][kMask ? j : 0]).x), -100));
        moved |= mx[nt][j] != m[nt][j] || ve[nt][j] != vexp[nt][j];
      }
    if (__any_sync(0xFFFFFFFFu, moved)) {
#pragma unroll
      for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int up = ve[nt][j] - vexp[nt][j];
          const float vshift = up > 100 ? 0.f : pow2i(-up);
          vexp[nt][j] = ve[nt][j];
          const float c = m[nt][j] == -INFINITY ? 0.f : ex2(m[nt][j] - mx[nt][j]), cv = c * vshift;
          m[nt][j] = mx[nt][j];
          l[nt][j] *= c; esum[nt][j] *= c; usum[nt][j] *= cv;
#pragma unroll
          for (int t = 0; t < 2 * kWords; ++t) { acc[nt][t][j] *= cv; acc[nt][t][2 + j] *= cv; }
        }
    }
    float vscale[kNT][2];
#pragma unroll
    for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
      for (int j = 0; j < 2; ++j) vscale[nt][j] = pow2i(min(13 - vexp[nt][j], 120));

    // ---- probabilities, and their products with the value codes
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
      float2 v0 = scale_floats<T>(vs[i][0]), v1 = scale_floats<T>(vs[i][1]);
      v0.y = fmaf(7.5f, v0.x, v0.y); v1.y = fmaf(7.5f, v1.x, v1.y);
      uint32_t b0[kNT], b1[kNT];
#pragma unroll
      for (int nt = 0; nt < kNT; ++nt) {
        float u[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const bool v = !kMask || ((seen >> ((i * kNT + nt) * 4 + e)) & 1u);
          const float p = v ? ex2(s[i][nt][e] - m[nt][e & 1]) : 0.f;
          l[nt][e & 1] += p;
          u[e] = p * ((e < 2 ? v0.x : v1.x) * vscale[nt][e & 1]);
          if (kMask) {
            if (!v) u[e] = 0.f;
            esum[nt][e & 1] += v ? p * (e < 2 ? v0.y : v1.y) : 0.f;
          } else {
            esum[nt][e & 1] = fmaf(p, e < 2 ? v0.y : v1.y, esum[nt][e & 1]);
          }
        }
        b0[nt] = transpose8x8(half2_bits(u[0], u[1]));
        b1[nt] = transpose8x8(half2_bits(u[2], u[3]));
        mma16816(usum[nt], kOnes, kOnes, kOnes, kOnes, b0[nt], b1[nt]);
      }
      uint32_t x[kWords], y[kWords];
      load_words<kWords>(stage + code_at[i] + v_off, x);
      load_words<kWords>(stage + code_at[i] + v_off + 4 * kDim, y);
#pragma unroll
      for (int k = 0; k < kWords; ++k) {
        const uint32_t xs = x[k] >> 8, ys = y[k] >> 8;
#pragma unroll
        for (int nt = 0; nt < kNT; ++nt) {
          mma16816(acc[nt][2 * k], x[k] & kLo, x[k] & kHi, y[k] & kLo, y[k] & kHi, b0[nt], b1[nt]);
          mma16816(acc[nt][2 * k + 1], xs & kLo, xs & kHi, ys & kLo, ys & kHi, b0[nt], b1[nt]);
        }
      }
    }
  };

  auto end_segment = [&](const Item& it) {
    const bool whole = !kCluster && from_start && it.last;
    // where the join finds the row block's parts: that of the first chunk (slot), that of the last (warp)
    if (!kCluster && lane == 0) {
      int* where = ends_at(a, plan, it.b, it.hk, it.rows0 / plan.rows_per_block);
      if (from_start) where[0] = 2 * w + later;
      if (it.last) where[1] = w;
    }
    if (kCluster) __syncwarp();                        // the part's sums take the place of its chunks
    float* slot = kCluster ? reinterpret_cast<float*>(ring) : slots_of(a) + (2 * w + later) * slot_floats(plan, kDim);
#pragma unroll
    for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        float lt = l[nt][j], et = esum[nt][j];
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) {
          lt += __shfl_xor_sync(0xFFFFFFFFu, lt, o);
          et += __shfl_xor_sync(0xFFFFFFFFu, et, o);
        }
        const int rr = nt * 8 + 2 * qd + j, r = it.rows0 + rr;
        if (rr >= plan.rows_per_block || r >= plan.rows) continue;
        const float back = pow2i(min(max(vexp[nt][j] - 13, -126), 127));
        const float add = et - 7.5f * usum[nt][j] * back, norm = whole ? (lt == 0.f ? 0.f : 1.f / lt) : 1.f;
        float o[kDim / 8];                             // values (kDim / 8) g .. of the row
#pragma unroll
        for (int t = 0; t < 2 * kWords; ++t) {
          o[2 * t] = (acc[nt][t][j] * 16777216.f * back + add) * norm;
          o[2 * t + 1] = (acc[nt][t][2 + j] * 1048576.f * back + add) * norm;
        }
        if (whole) {
          const int i_q = r / plan.group;
          T* out = reinterpret_cast<T*>(a.o) + ((int64_t)it.b * a.n_q + i_q) * a.ld_o +
                   (int64_t)(it.hk * plan.group + r - i_q * plan.group) * kDim + g * (kDim / 8);
#pragma unroll
          for (int i = 0; i < kDim / 64; ++i)
            *reinterpret_cast<uint4*>(out + 8 * i) =
                make_uint4(pair_bits<T>(o[8 * i], o[8 * i + 1]), pair_bits<T>(o[8 * i + 2], o[8 * i + 3]),
                           pair_bits<T>(o[8 * i + 4], o[8 * i + 5]), pair_bits<T>(o[8 * i + 6], o[8 * i + 7]));
        } else {
          float* row = slot + rr * (kDim + 4);
#pragma unroll
          for (int i = 0; i < kDim / 32; ++i)
            *reinterpret_cast<float4*>(row + g * (kDim / 8) + 4 * i) = make_float4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
          if (g == 0) *reinterpret_cast<float2*>(row + kDim) = make_float2(m[nt][j], lt);
        }
      }
    later = true;
  };

  // The copies of an item have come (and, all lanes being here, its predecessor's stage is free).  False: the wait ran out.
  auto arrived = [&](int item, uint32_t limit) -> bool {
    const uint32_t bar = bar_addr + 8 * (item % kStages), parity = (uint32_t)(item / kStages) & 1u;
    if (limit && __all_sync(0xFFFFFFFFu, tc::mbar_try_wait(bar, parity))) return true;
    bool ok = false;
    unsigned long long t0 = 0;
    for (uint32_t i = 0; i < limit && !ok; ++i) {
      ok = tc::mbar_try_wait(bar, parity);
      if ((i & 255u) == 255u) {
        const unsigned long long now = tc::global_ns();
        if (t0 == 0) t0 = now;
        else if (now - t0 > tc::kWaitNs) break;
      }
    }
    return __all_sync(0xFFFFFFFFu, ok);
  };
  __syncwarp();
  if (!kCluster || items > 0) begin_segment(items_of[0]);   // while the first chunk is on its way
  bool fresh = false;
  for (int item = 0; item < items; ++item) {
    if (!arrived(item, polls)) {                       // the copies did not come: reported, and the rows that miss them become NaN
      if (lane == 0) set_status(a.ws, BL_ERR_TIMEOUT);
      for (int i = item; i < min(issued, items); ++i) arrived(i, tc::kSpinLimit);   // those in flight end before the CTA does (bounded)
      if (!kCluster) {
        lose_items<T, kDim>(a, plan, item, later, from_start, fresh);
        return;
      }
      __syncwarp();                                    // the part's sums take the place of its chunks, where the copies have ended
      if (lane < plan.rows_per_block)
        *reinterpret_cast<float2*>(reinterpret_cast<float*>(ring) + lane * (kDim + 4) + kDim) = make_float2(-INFINITY, __int_as_float(0x7FC00000));
      break;
    }
    const Item it = items_of[item % kStages];
    issue();
    if (fresh) begin_segment(it);
    fresh = it.last;
    const bool all_see = it.there == (1 << subs) - 1 && it.t0 + kChunk - 1 <= it.len - back_first &&
                         (a.window == 0 || it.len - back_last - it.t0 < a.window || it.t0 + kChunk <= a.sinks);
    const char* stage = ring + (item % kStages) * kStageBytes;
    if (all_see) chunk(stage, it, std::false_type{});
    else chunk(stage, it, std::true_type{});
    if (it.last || item + 1 == items) end_segment(it);
  }
  if (!kCluster) return;

  // ---- the parts of the CTA's warps become one, then those of the cluster's CTAs
  constexpr int kRow = kDim + 4;                       // a row's sums, its maximum, the sum of its probabilities
  float* joined = reinterpret_cast<float*>(smem + kWarps * kStages * (kStageBytes + (int)sizeof(Item) + 8));
  if (items == 0 && lane < plan.rows_per_block)        // nothing
    *reinterpret_cast<float2*>(reinterpret_cast<float*>(ring) + lane * kRow + kDim) = make_float2(-INFINITY, 0.f);
  __syncthreads();
  const int rows0 = ahead.blk * plan.rows_per_block, rows = min(plan.rows_per_block, plan.rows - rows0);
  for (int e = 2 * threadIdx.x; e < rows * kDim; e += kWarps * 64) {
    const int rr = e / kDim, d = e & (kDim - 1);
    const float* part = reinterpret_cast<const float*>(smem) + rr * kRow;
    float top = -INFINITY, l = 0.f;
    float2 v = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < kWarps; ++i) top = fmaxf(top, part[i * (kStages * kStageBytes / 4) + kDim]);
#pragma unroll
    for (int i = 0; i < kWarps; ++i) {
      const float* x = part + i * (kStages * kStageBytes / 4);
      if (sees_nothing(x[kDim], x[kDim + 1])) continue;
      const float c = ex2(x[kDim] - top);
      l = fmaf(x[kDim + 1], c, l);
      v.x = fmaf(x[d], c, v.x); v.y = fmaf(x[d + 1], c, v.y);
    }
    *reinterpret_cast<float2*>(joined + rr * kRow + d) = v;
    if (d == 0) *reinterpret_cast<float2*>(joined + rr * kRow + kDim) = make_float2(top, l);
  }
  __syncwarp();
  cluster_meet();
  const int ctas = 1 << plan.cluster_log2;
  for (int e = 2 * (rank * kWarps * 32 + threadIdx.x); e < rows * kDim; e += ctas * kWarps * 64) {
    const int rr = e / kDim, d = e & (kDim - 1), r = rows0 + rr, i_q = r / plan.group;
    float2 stat[kMostCluster], x[kMostCluster];
#pragma unroll
    for (int i = 0; i < kMostCluster; ++i) {
      stat[i] = i < ctas ? peer_float2(joined + rr * kRow + kDim, i) : make_float2(-INFINITY, 0.f);
      x[i] = i < ctas ? peer_float2(joined + rr * kRow + d, i) : make_float2(0.f, 0.f);
    }
    float top = -INFINITY, l = 0.f;
    float2 v = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < kMostCluster; ++i) top = fmaxf(top, stat[i].x);
#pragma unroll
    for (int i = 0; i < kMostCluster; ++i) {
      if (sees_nothing(stat[i].x, stat[i].y)) continue;
      const float c = ex2(stat[i].x - top);
      l = fmaf(stat[i].y, c, l);
      v.x = fmaf(x[i].x, c, v.x); v.y = fmaf(x[i].y, c, v.y);
    }
    const float norm = l == 0.f ? 0.f : 1.f / l;
    T* out = reinterpret_cast<T*>(a.o) + ((int64_t)ahead.b * a.n_q + i_q) * a.ld_o + (int64_t)(ahead.hk * plan.group + r - i_q * plan.group) * kDim + d;
    *reinterpret_cast<uint32_t*>(out) = pair_bits<T>(v.x * norm, v.y * norm);
  }
  __syncwarp();
  cluster_meet();                                      // the others have read this CTA's sums
}

template <int kVals> __device__ __forceinline__ void load_values(const float* p, float (&x)[kVals]);
template <> __device__ __forceinline__ void load_values<4>(const float* p, float (&x)[4]) {
  const float4 v = *reinterpret_cast<const float4*>(p);
  x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
}
template <> __device__ __forceinline__ void load_values<2>(const float* p, float (&x)[2]) {
  const float2 v = *reinterpret_cast<const float2*>(p);
  x[0] = v.x; x[1] = v.y;
}

// The parts of one row of the result.
template <typename T> struct JoinRow {
  const float* first;                                  // the first part's sums; the others lie `stride` apart behind
  const float* others;                                 // that of part i > 0 at others + i * stride
  int64_t stride;
  int parts;                                           // 0: an empty sequence; 1: written already, or nothing to write
  T* out;
  __device__ __forceinline__ const float* part(int i) const { return i == 0 ? first : others + i * stride; }
};
template <typename T, int kDim> __device__ __forceinline__ JoinRow<T> join_row(const Kv4AttnArgs& a, const Plan& plan, int64_t index) {
  JoinRow<T> x;
  x.parts = 1;
  x.first = x.others = nullptr; x.stride = 0; x.out = nullptr;
  const int bh = (int)((uint32_t)index / (uint32_t)plan.rows_per_block), rr = (int)(index - (int64_t)bh * plan.rows_per_block);
  const int b = bh / plan.heads_blocks, hb = bh - b * plan.heads_blocks;
  if (b >= a.batch) return x;
  const int hk = hb / plan.blocks, r = (hb - hk * plan.blocks) * plan.rows_per_block + rr, i_q = r / plan.group;
  if (r >= plan.rows) return x;
  x.out = reinterpret_cast<T*>(a.o) + ((int64_t)b * a.n_q + i_q) * a.ld_o + (int64_t)(hk * plan.group + r - i_q * plan.group) * kDim;
  const int2 ends = *reinterpret_cast<const int2*>(ends_of(a, plan) + 2 * (int64_t)bh);
  if (make_seq(a, b).chunks == 0) {
    x.parts = 0;
    return x;
  }
  const int w0 = ends.x >> 1, parts = part_count(ends.x, ends.y, plan.parts);
  if (parts == 0) return x;                            // cannot be: the first kernel's warps end every list, also one whose copies did not come
  // the first part may be in its warp's second slot; the others are in first slots
  x.parts = parts;
  x.stride = 2 * slot_floats(plan, kDim);
  x.others = slots_of(a) + w0 * x.stride + rr * (kDim + 4);
  x.first = x.others + (ends.x & 1) * (x.stride / 2);
  return x;
}

// Joins a row by a CTA.  All maxima and sums are loaded at once; then the parts' values are summed, kLoads parts of a warp in flight.
template <int kDim, int kWarps> struct JoinSpace { float2 stats[kMaxSms * kMostWarps]; float sums[kWarps][kDim], tops[kWarps], totals[kWarps]; };
template <typename T, int kDim, int kWarps> __device__ __forceinline__ void join_by_cta(const JoinRow<T>& x, JoinSpace<kDim, kWarps>& sh) {
  constexpr int kVals = kDim / 32, kLoads = kWarps > 8 ? 4 : 8;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  float top = -INFINITY;
  for (int i = threadIdx.x; i < x.parts; i += kWarps * 32) {
    const float2 st = *reinterpret_cast<const float2*>(x.part(i) + kDim);
    sh.stats[i] = st;
    top = fmaxf(top, st.x);
  }
  top = warp_max(top);
  if (lane == 0) sh.tops[warp] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kWarps; ++i) top = fmaxf(top, sh.tops[i]);
  float l = 0.f, v[kVals] = {};
  for (int base = warp; base < x.parts; base += kLoads * kWarps) {
    float y[kLoads][kVals];
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      const int i = base + u * kWarps;
      if (i < x.parts) load_values<kVals>(x.part(i) + lane * kVals, y[u]);
    }
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      const int i = base + u * kWarps;
      if (i >= x.parts) break;
      const float2 st = sh.stats[i];
      if (sees_nothing(st.x, st.y)) continue;
      const float c = ex2(st.x - top);
      l = fmaf(st.y, c, l);
#pragma unroll
      for (int e = 0; e < kVals; ++e) v[e] = fmaf(y[u][e], c, v[e]);
    }
  }
  if (lane == 0) sh.totals[warp] = l;
#pragma unroll
  for (int e = 0; e < kVals; ++e) sh.sums[warp][lane * kVals + e] = v[e];
  __syncthreads();
  for (int d = threadIdx.x; d < kDim; d += kWarps * 32) {
    float ls = 0.f, vs = 0.f;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) { ls += sh.totals[i]; vs += sh.sums[i][d]; }
    x.out[d] = out_cast<T>(ls == 0.f ? 0.f : vs / ls);
  }
}

// Joins the parts of the rows whose chunks went to more than one warp.  kPerWarp: a warp per row (one of more than 32 parts is
// left to the whole CTA), for many rows of mostly few parts; else a CTA per row.
template <typename T, int kDim, int kWarps, bool kPerWarp>
__global__ void __launch_bounds__(kWarps * 32) attention_kv4_join_kernel(Kv4AttnArgs a, Plan plan) {
  __shared__ JoinSpace<kDim, kWarps> space;
  __shared__ JoinRow<T> rows[kPerWarp ? kWarps : 1];
  constexpr int kVals = kDim / 32, kLoads = 8;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  pdl_launch_dependents();
  pdl_wait();
  const JoinRow<T> x = join_row<T, kDim>(a, plan, kPerWarp ? (int64_t)blockIdx.x * kWarps + warp : (int64_t)blockIdx.x);
  if (x.parts == 0 && (kPerWarp || warp == 0)) {
    for (int d = lane; d < kDim; d += 32) x.out[d] = out_cast<T>(0.f);
  }
  if (!kPerWarp) {
    if (x.parts > 1) join_by_cta<T, kDim, kWarps>(x, space);
    return;
  }
  if (x.parts > 1 && x.parts <= 32) {
    const float2 st = lane < x.parts ? *reinterpret_cast<const float2*>(x.part(lane) + kDim) : make_float2(-INFINITY, 0.f);
    const bool none = sees_nothing(st.x, st.y);
    const float top = warp_max(st.x), c = none ? 0.f : ex2(st.x - top);
    const float l = warp_sum(none ? 0.f : st.y * c);
    const unsigned takes = __ballot_sync(0xFFFFFFFFu, !none);
    float v[kVals] = {};
    for (int base = 0; base < x.parts; base += kLoads) {
      float y[kLoads][kVals];
#pragma unroll
      for (int u = 0; u < kLoads; ++u)
        if (base + u < x.parts) load_values<kVals>(x.part(base + u) + lane * kVals, y[u]);
#pragma unroll
      for (int u = 0; u < kLoads; ++u) {
        const float cu = __shfl_sync(0xFFFFFFFFu, c, (base + u) & 31);
        if (base + u >= x.parts || !((takes >> ((base + u) & 31)) & 1u)) continue;
#pragma unroll
        for (int e = 0; e < kVals; ++e) v[e] = fmaf(y[u][e], cu, v[e]);
      }
    }
#pragma unroll
    for (int e = 0; e < kVals; ++e) x.out[lane * kVals + e] = out_cast<T>(l == 0.f ? 0.f : v[e] / l);
  }
  if (lane == 0) rows[warp] = x;
  if (!__syncthreads_or(x.parts > 32)) return;
  for (int i = 0; i < kWarps; ++i)
    if (rows[i].parts > 32) {
      join_by_cta<T, kDim, kWarps>(rows[i], space);
      __syncthreads();
    }
}

cudaError_t sm_count(int dev, int* n) {
  static std::atomic<int> known[64];
  if (dev < 64 && (*n = known[dev].load(std::memory_order_relaxed)) > 0) return cudaSuccess;
  const cudaError_t e = cudaDeviceGetAttribute(n, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return e;
  if (*n > kMaxSms) *n = kMaxSms;
  if (dev < 64) known[dev].store(*n, std::memory_order_relaxed);
  return cudaSuccess;
}

template <int kDim, int kNT, int kWarps, int kStages, bool kCluster> constexpr int smem_bytes() {
  constexpr int kSmem = kWarps * kStages * (kChunk * (kDim + 8) + (int)sizeof(Item) + 8) + (kCluster ? kNT * 8 * (kDim + 4) * 4 : 0);
  static_assert(kSmem <= 232448, "exceeds the shared memory of one CTA");
  static_assert(!kCluster || kNT * 8 * (kDim + 4) * 4 <= kStages * kChunk * (kDim + 8), "a part's sums exceed the place of its chunks");
  return kSmem;
}
// Lets the kernel have its shared memory, once per device.
template <typename T, int kDim, int kNT, int kWarps, int kStages, bool kCluster> cudaError_t allow_smem(int dev) {
  static std::atomic<uint64_t> ready{0};
  if (dev < 64 && ((ready.load(std::memory_order_relaxed) >> dev) & 1)) return cudaSuccess;
  const cudaError_t e = cudaFuncSetAttribute(attention_kv4_kernel<T, kDim, kNT, kWarps, kStages, kCluster>,
                                             cudaFuncAttributeMaxDynamicSharedMemorySize, smem_bytes<kDim, kNT, kWarps, kStages, kCluster>());
  if (e == cudaSuccess && dev < 64) ready.fetch_or(1ull << dev, std::memory_order_relaxed);
  return e;
}
inline uint32_t wait_polls() {
  const long long dbg = g_debug_wait_polls.load(std::memory_order_relaxed);
  return dbg < 0 ? tc::kSpinLimit : (uint32_t)(dbg < (long long)tc::kSpinLimit ? dbg : tc::kSpinLimit);
}

// A cluster per list, if all of them fit the GPU at once and have at most four chunks per warp; *done says whether.  Of the
// sizes that fit, the smallest that leaves a warp no more than one chunk, else the largest.  Against the cut list and the join
// (us, 128-wide heads): 1 x 1000 tokens, 16 heads 6.3 / 8.3; 4 x 4000, 8 heads of 4 rows 8.9 / 13.0; 1 x 8000, 8 heads of 16 rows
// 13.0 / 14.7; 1 x 16000, 16 heads (8 chunks per warp) 18.7 / 16.1; clusters that do not fit at once 11.9 / 9.5 (1 x 4000, 16 heads).
template <typename T, int kDim, int kNT>
cudaError_t launch_clusters(const Kv4AttnArgs& a, int dev, int64_t lists, int64_t chunks, cudaStream_t s, bool* done) {
  static std::atomic<int> known[64][kMostClusterLog2 + 1];     // clusters of 2^i CTAs that fit, and 1
  const auto kernel = attention_kv4_kernel<T, kDim, kNT, 8, 2, true>;
  constexpr int kSmem = smem_bytes<kDim, kNT, 8, 2, true>();
  *done = false;
  int size = -1;
  for (int i = 0; i <= kMostClusterLog2 && (size < 0 || chunks > 8 << size); ++i) {
    int fit = dev < 64 ? known[dev][i].load(std::memory_order_relaxed) - 1 : -1;
    if (fit < 0) {
      cudaError_t e = allow_smem<T, kDim, kNT, 8, 2, true>(dev);
      if (e == cudaSuccess) e = max_clusters(kernel, 1u << i, 256, kSmem, &fit);
      if (e != cudaSuccess) return e;
      if (dev < 64) known[dev][i].store(fit + 1, std::memory_order_relaxed);
    }
    if (lists <= fit && lists << i <= kMaxSms) size = i;       // (no more warps than the workspace has status words for)
  }
  if (size < 0 || chunks > kClusterChunks * 8 << size) return cudaSuccess;
  *done = true;
  const Plan plan = make_plan(a.n_q, a.heads, a.cache.kv_heads, a.cache.page_size, 8 << size, size);
  return launch_pdl_clusters(kernel, (unsigned)lists << size, 1u << size, 256, kSmem, s, a, plan, wait_polls());
}

template <typename T, int kDim, int kNT, int kWarps, int kStages>
cudaError_t launch_rows(const Kv4AttnArgs& a, int dev, int sms, cudaStream_t s) {
  constexpr int kSmem = smem_bytes<kDim, kNT, kWarps, kStages, false>();
  const auto kernel = attention_kv4_kernel<T, kDim, kNT, kWarps, kStages, false>;
  cudaError_t e = allow_smem<T, kDim, kNT, kWarps, kStages, false>(dev);
  if (e != cudaSuccess) return e;
  const uint32_t polls = wait_polls();
  const Plan plan = make_plan(a.n_q, a.heads, a.cache.kv_heads, a.cache.page_size, sms * kWarps);
  e = launch_pdl(kernel, (unsigned)sms, kWarps * 32, kSmem, s, a, plan, polls);
  if (e != cudaSuccess) return e;
  // A CTA per row, of 32 warps while each has an SM to itself (32000 tokens, 8 heads, 4 rows: 17.3 us against 23.8 with 8; with
  // more rows 16 warps already lose, 14.5 against 12.0 at 16 x 1000 tokens).  Many rows have few parts each, and get a warp (256 x
  // 1000 tokens, 8 heads, 4 rows: 70 us against 93; 256 x 60: 18 against 30; but 8 x 16000, 256 rows: 40 against 34).
  const int64_t rows = (int64_t)a.batch * plan.heads_blocks * plan.rows_per_block;
  if (rows <= sms) return launch_pdl(attention_kv4_join_kernel<T, kDim, 32, false>, (unsigned)rows, 1024, 0, s, a, plan);
  if (rows <= kCtaRows * sms) return launch_pdl(attention_kv4_join_kernel<T, kDim, 8, false>, (unsigned)rows, 256, 0, s, a, plan);
  return launch_pdl(attention_kv4_join_kernel<T, kDim, 8, true>, (unsigned)((rows + 7) / 8), 256, 0, s, a, plan);
}

// Longer or more lists.  Up to 8 query rows: 12 warps with two chunks each keep the SM busier (32 x 8192 tokens, 8 heads, 4 rows:
// 45.4 us against 49.3 with 8 warps and three chunks), but the next kernel finds no room beside them before they end, which costs
// a short list 1 to 2 us (64 x 120 tokens, 16 heads: 18.5 against 16.2), so lists of at most two chunks per warp take 8.  More
// rows: 8 warps, whose 255 registers hold the second tile of rows (12: spills, 116 us against 83 for 2 x 150001 tokens).
template <typename T, int kDim>
cudaError_t launch_dim(const Kv4AttnArgs& a, cudaStream_t s) {
  const int64_t rows = (int64_t)a.n_q * (a.heads / a.cache.kv_heads);
  int64_t tokens = a.max_pages * a.cache.page_size;
  if (a.window > 0) tokens = std::min<int64_t>(tokens, (int64_t)a.window + a.sinks + a.n_q + 2 * kChunk);
  const int64_t chunks = (tokens + kChunk - 1) / kChunk, lists = (int64_t)a.batch * a.cache.kv_heads * (rows <= 8 ? 1 : (rows + 15) / 16);
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = sm_count(dev, &sms);
  if (e != cudaSuccess) return e;
  bool done = false;
  e = rows > 8 ? launch_clusters<T, kDim, 2>(a, dev, lists, chunks, s, &done) : launch_clusters<T, kDim, 1>(a, dev, lists, chunks, s, &done);
  if (done || e != cudaSuccess) return e;
  if (rows > 8) return launch_rows<T, kDim, 2, 8, 3>(a, dev, sms, s);
  return chunks * lists <= 2 * 8 * 148 ? launch_rows<T, kDim, 1, 8, 3>(a, dev, sms, s) : launch_rows<T, kDim, 1, 12, 2>(a, dev, sms, s);
}

template <typename T>
cudaError_t launch_type(const Kv4AttnArgs& a, cudaStream_t s) {
  return a.cache.head_dim == 64 ? launch_dim<T, 64>(a, s) : launch_dim<T, 128>(a, s);
}

}  // namespace

size_t attention_kv4_ws_bytes(int batch, int n_q, int heads, int kv_heads, int head_dim) {
  const Plan p = make_plan(n_q, heads, kv_heads, 16, 1);
  return batch == 0 ? 0 : kStatusBytes + (size_t)kMaxSms * kMostWarps * 2 * (size_t)slot_floats(p, head_dim) * sizeof(float) +
                              (size_t)batch * (size_t)p.heads_blocks * 2 * sizeof(int);
}

cudaError_t launch_attention_kv4(const Kv4AttnArgs& a, cudaStream_t s) {
  return a.cache.dtype == BL_F16 ? launch_type<__half>(a, s) : launch_type<__nv_bfloat16>(a, s);
}

}  // namespace bl
