// Attention of prompts with a sliding window and sinks (bitlinear_attention_window):
//   o_i = sum_j p_ij v_j / sum_j p_ij,  p_ij = e^(scale q_i . k_j - max),  j visible from i.
//
// A CTA owns a tile of 128 query rows of one head; two CTAs share an SM, so that one's softmax, copies, start and end
// run beside the other's products.  Keys and values pass through shared memory in tiles of 64; tiles that no row sees
// (after the rows, or between the sinks and the window) are not loaded.  Per key tile two products of 128 x 64 x kDim
// run on the tcgen05 tensor cores,
//   S = Q K^T   both operands in shared memory (TMA, 128-byte swizzle), S in tensor memory (fp32),
//   O += P V    P in tensor memory as 16-bit numbers, over S; V as it lies in memory (its rows are the
//               contraction, so the descriptor says MN-major); O in tensor memory (fp32).
// There are two places for S: while the softmax works on S(i), S(i+1) is being formed or is there already.  The products
// run in issue order S(i+1), PV(i), S(i+2), .., which is what keeps S(i+2) from overwriting P(i).  With one place of 128
// keys the softmax (1900 clocks) and the products (1700 with their latencies) took turns: 1.6 times as long.  Two query
// tiles in one CTA per SM share the loads of a group's keys, but run in step: 3 % faster on one prompt of 8192 with a
// window of 4096 (372 against 380 us), 5 to 20 % slower on shorter prompts and windows and with heads of 64.
//
// Precision.  Scores, statistics and sums in fp32.  The probabilities are rounded to the type of V, which the tensor core wants of
// both operands; their sum is that of the numbers before the rounding.  Against products in fp32 throughout that raises the error
// from 1.9e-4 to 2.6e-4 of the result (fp16, 4 x 2048 tokens) and from 1.5e-3 to 2.0e-3 (bf16, 8192), half of it the output's own.
//
// Roles: warps 0-3 the softmax (a thread owns a query row: no shuffles), warp 4 issues the products, warp 5 the
// copies.  The running maximum moves only when a row's maximum grew by more than 2^8: O is then rescaled in tensor
// memory, which is rare; else probabilities of up to 2^8 do no harm (they are formed at 2^7 times their size, 2^15 at
// most, so that the smallest fp16 probability is 2^-31 of a row's largest or less).
//
// Invisible places.  A masked score is replaced, so keys there may be anything.  A value there meets a probability
// of 0, but 0 x NaN is NaN: values behind a sequence's end are cleared in shared memory, and a row whose result is not
// finite although its sum is, is computed again by one warp from the visible places alone (window_row).  Finite values
// never take that path.
//
// Every wait is bounded.  If one runs out, the CTA's rows are computed by window_row too and the event is
// counted (bitlinear_debug_window_fallbacks): the result is the same up to rounding, only late.
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "tc_common.cuh"

namespace bl {

namespace {

using namespace tc;

__device__ unsigned int g_window_fallbacks;      // CTAs whose waits ran out, since last asked

// Rows of one sequence in q / o and in k / v.
struct SeqRows { int q0, nq, k0, nk; };
__device__ __forceinline__ SeqRows seq_rows(const WindowArgs& a, int b) {
  SeqRows r;
  if (a.cu_q) {
    r.q0 = min(max(a.cu_q[b], 0), (int)a.rows_q);
    r.nq = min(min(max(a.cu_q[b + 1], r.q0), (int)a.rows_q) - r.q0, (int)a.seq_q);
    r.k0 = min(max(a.cu_k[b], 0), (int)a.rows_k);
    r.nk = min(min(max(a.cu_k[b + 1], r.k0), (int)a.rows_k) - r.k0, (int)a.seq_k);
  } else {
    r.q0 = b * (int)a.seq_q; r.nq = (int)a.seq_q;
    r.k0 = b * (int)a.seq_k; r.nk = (int)a.seq_k;
  }
  return r;
}

// Query row i (of r.nq) of head h, by one warp.
template <typename T, int kDim>
__device__ void window_row(const WindowArgs& a, const SeqRows& r, int i, int h) {
  constexpr int kVals = kDim / 32;
  const int lane = threadIdx.x & 31, hk = h / (a.heads / a.kv_heads), pos = r.nk - r.nq + i;
  const T* q = reinterpret_cast<const T*>(a.q) + (int64_t)(r.q0 + i) * a.ld_q + (int64_t)h * kDim + lane * kVals;
  const T* k = reinterpret_cast<const T*>(a.k) + (int64_t)r.k0 * a.ld_k + (int64_t)hk * kDim + lane * kVals;
  const T* v = reinterpret_cast<const T*>(a.v) + (int64_t)r.k0 * a.ld_v + (int64_t)hk * kDim + lane * kVals;
  float qv[kVals], acc[kVals];
#pragma unroll
  for (int e = 0; e < kVals; ++e) { qv[e] = in_cast(q[e]); acc[e] = 0.f; }
  float m = -INFINITY, l = 0.f;
  for (int j = 0; j <= pos; ++j) {
    if (a.window > 0 && pos - j >= a.window && j >= a.sinks) continue;
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < kVals; ++e) s = fmaf(qv[e], in_cast(k[(int64_t)j * a.ld_k + e]), s);
    s = warp_sum(s) * a.scale;
    const float top = fmaxf(m, s), c = m == -INFINITY ? 0.f : expf(m - top), p = expf(s - top);
    m = top;
    l = l * c + p;
#pragma unroll
    for (int e = 0; e < kVals; ++e) acc[e] = acc[e] * c + p * in_cast(v[(int64_t)j * a.ld_v + e]);
  }
  T* o = reinterpret_cast<T*>(a.o) + (int64_t)(r.q0 + i) * a.ld_o + (int64_t)h * kDim + lane * kVals;
#pragma unroll
  for (int e = 0; e < kVals; ++e) o[e] = out_cast<T>(l == 0.f ? 0.f : acc[e] / l);
}

constexpr int kRows = 128;                       // query rows per CTA
constexpr int kKeys = 64;                        // keys per tile
constexpr int kMostSlots = 8;                    // key or value tiles in shared memory
constexpr int kThreads = 192, kIssuer = 4, kCopier = 5;
constexpr int kTmemCols = 256;                   // two places for S (64 columns each), O (128)
constexpr float kMoveLog2 = 8.f;                 // growth of a row's maximum that is let pass
constexpr float kLiftLog2 = 7.f;                 // probabilities are formed 2^7 times their size

struct Ctl {
  unsigned long long q_full, kv_full[kMostSlots], kv_empty[kMostSlots], s_full[2], p_ready[2], o_done[2], drain;
  uint32_t tmem_base;
  int abort_flag;
};

// Bounded wait like mbar_wait, with the number of polls from the launch (tests shorten it).
__device__ __forceinline__ bool wait_for(unsigned long long* bar, uint32_t parity, volatile int* abort_flag, uint32_t polls) {
  const uint32_t b = smem_u32(bar);
  unsigned long long t0 = 0;                     // the clock is read only once a wait has become long
  for (uint32_t it = 0; it < polls; ++it) {
    if (mbar_try_wait(b, parity)) return true;
    if ((it & 255u) == 255u) {
      if (*abort_flag) return false;
      const unsigned long long now = global_ns();
      if (t0 == 0) t0 = now;
      else if (now - t0 > kWaitNs) break;
    }
  }
  *abort_flag = 1;
  return false;
}

// The same by a whole warp, with one answer for all of it.
__device__ __forceinline__ bool wait_warp(unsigned long long* bar, uint32_t parity, volatile int* abort_flag, uint32_t polls) {
  if (polls && __all_sync(0xFFFFFFFFu, mbar_try_wait(smem_u32(bar), parity))) return true;
  return __all_sync(0xFFFFFFFFu, wait_for(bar, parity, abort_flag, polls));
}

// kind::f16 instruction descriptor: fp32 sums, fp16 or bf16 operands, M = 128.
template <typename T> __host__ __device__ constexpr uint32_t idesc(int n, bool b_mn_major) {
  const uint32_t type = std::is_same<T, __half>::value ? 0u : 1u;
  return (1u << 4) | (type << 7) | (type << 10) | ((b_mn_major ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) | (8u << 24);
}
// K-major tile of 128-byte rows: smem_desc_sw128.  MN-major: rows of 64 values along N, groups of 8 rows (of the
// contraction) 1024 bytes apart, the next 64 values along N one sub-tile (kKeys rows) further.
__device__ __forceinline__ uint64_t desc_mn(uint32_t addr) {
  uint64_t d = 0;
  d |= (uint64_t)((addr & 0x3FFFFu) >> 4);
  d |= (uint64_t)((kKeys * 128) >> 4) << 16;
  d |= (uint64_t)(1024 >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}
// The instructions of the tensor core, issued by the lane whose `on` is set.  The whole warp executes them: in code that one
// lane runs alone the operands cannot stay in the uniform registers that the instruction reads, and moving them there cost
// more than the product itself (85 clocks per product of 64; the pair of tiles took 4520 clocks instead of 3300).
__device__ __forceinline__ uint32_t elect() {
  uint32_t on;
  asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xFFFFFFFF;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(on));
  return on;
}
__device__ __forceinline__ void mma_ss(uint32_t on, uint32_t d, uint64_t a, uint64_t b, uint32_t id, uint32_t accumulate) {
  asm volatile("{\n.reg .pred p, e;\nsetp.ne.b32 p, %4, 0;\nsetp.ne.b32 e, %5, 0;\n"
               "@e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}"
               ::"r"(d), "l"(a), "l"(b), "r"(id), "r"(accumulate), "r"(on) : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t on, uint32_t d, uint32_t a, uint64_t b, uint32_t id, uint32_t accumulate) {
  asm volatile("{\n.reg .pred p, e;\nsetp.ne.b32 p, %4, 0;\nsetp.ne.b32 e, %5, 0;\n"
               "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}"
               ::"r"(d), "r"(a), "l"(b), "r"(id), "r"(accumulate), "r"(on) : "memory");
}
__device__ __forceinline__ void commit(uint32_t on, unsigned long long* bar) {
  asm volatile("{\n.reg .pred e;\nsetp.ne.b32 e, %1, 0;\n"
               "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}" ::"r"(smem_u32(bar)), "r"(on) : "memory");
}
// 32 columns of this warp's 32 lanes, without the wait.
__device__ __forceinline__ void ld32(uint32_t taddr, float* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]), "=f"(r[8]), "=f"(r[9]),
        "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15]), "=f"(r[16]), "=f"(r[17]), "=f"(r[18]),
        "=f"(r[19]), "=f"(r[20]), "=f"(r[21]), "=f"(r[22]), "=f"(r[23]), "=f"(r[24]), "=f"(r[25]), "=f"(r[26]), "=f"(r[27]),
        "=f"(r[28]), "=f"(r[29]), "=f"(r[30]), "=f"(r[31])
      : "r"(taddr));
}
// Waits for the loads above; r, what one of them loaded, is an operand so that no use of it moves ahead of the wait.
__device__ __forceinline__ void ld_wait(float* r) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+f"(r[0]), "+f"(r[1]), "+f"(r[2]), "+f"(r[3]), "+f"(r[4]), "+f"(r[5]), "+f"(r[6]), "+f"(r[7]), "+f"(r[8]), "+f"(r[9]),
                 "+f"(r[10]), "+f"(r[11]), "+f"(r[12]), "+f"(r[13]), "+f"(r[14]), "+f"(r[15]), "+f"(r[16]), "+f"(r[17]), "+f"(r[18]),
                 "+f"(r[19]), "+f"(r[20]), "+f"(r[21]), "+f"(r[22]), "+f"(r[23]), "+f"(r[24]), "+f"(r[25]), "+f"(r[26]), "+f"(r[27]),
                 "+f"(r[28]), "+f"(r[29]), "+f"(r[30]), "+f"(r[31])
               :: "memory");
}
__device__ __forceinline__ void st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
template <typename R> __device__ __forceinline__ void st32(uint32_t taddr, const R* r) {
  static_assert(sizeof(R) == 4, "32-bit columns");
  const uint32_t* u = reinterpret_cast<const uint32_t*>(r);
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
      "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
      ::"r"(taddr), "r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]), "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7]), "r"(u[8]), "r"(u[9]),
        "r"(u[10]), "r"(u[11]), "r"(u[12]), "r"(u[13]), "r"(u[14]), "r"(u[15]), "r"(u[16]), "r"(u[17]), "r"(u[18]), "r"(u[19]),
        "r"(u[20]), "r"(u[21]), "r"(u[22]), "r"(u[23]), "r"(u[24]), "r"(u[25]), "r"(u[26]), "r"(u[27]), "r"(u[28]), "r"(u[29]),
        "r"(u[30]), "r"(u[31]) : "memory");
}
// Two fp32 numbers in one 64-bit register, and the instructions that work on both.
using f32x2 = unsigned long long;
__device__ __forceinline__ f32x2 pair(float a, float b) { f32x2 r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ float2 halves(f32x2 r) { float2 v; asm("mov.b64 {%0, %1}, %2;" : "=f"(v.x), "=f"(v.y) : "l"(r)); return v; }
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) { f32x2 r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) { f32x2 r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ float max3(float a, float b, float c) { float r; asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c)); return r; }
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
template <typename T> __device__ __forceinline__ uint32_t pack2(float lo, float hi);
template <> __device__ __forceinline__ uint32_t pack2<__half>(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// What a CTA works on; every role derives the same.
struct Job {
  SeqRows r;
  int head, row0, rows, pos0, pos1;              // head, first query row of the sequence, rows (0: none), their positions
  int sink_tiles, first, count;                  // key tiles: those of the sinks, then `first` on
  int clean_from, clean_to;                      // those that every row sees as a whole (tiles of nothing but sinks are not counted in)
  __device__ __forceinline__ int key0(int j) const { return (j < sink_tiles ? j : first + j - sink_tiles) * kKeys; }
};
// The heads of a group lie side by side, so that they find their keys in L2; within a sequence (with equal lengths: in the
// whole batch) the blocks with the most keys come first.  Packed sequences have as many blocks as their rows need, found by
// a sum over the batch: a bound of the lengths far above most of them costs nothing.  By whole warps, each for itself.
__device__ __forceinline__ Job make_job(const WindowArgs& a) {
  Job w;
  const int unit = blockIdx.x / a.heads, lane = threadIdx.x & 31;
  int b = a.batch, blk = 0;
  w.head = blockIdx.x - unit * a.heads;
  if (!a.cu_q) {
    b = unit % a.batch;
    blk = (int)((a.seq_q + kRows - 1) / kRows) - 1 - unit / a.batch;
  } else {
    int before = 0;
    for (int base = 0; base < a.batch; base += 32) {
      const int n = base + lane < a.batch ? (seq_rows(a, base + lane).nq + kRows - 1) / kRows : 0;
      int upto = n;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int up = __shfl_up_sync(0xFFFFFFFFu, upto, o);
        if (lane >= o) upto += up;
      }
      const unsigned past = __ballot_sync(0xFFFFFFFFu, before + upto > unit);
      if (past) {
        const int f = __ffs(past) - 1;
        b = base + f;
        blk = before + __shfl_sync(0xFFFFFFFFu, upto, f) - 1 - unit;
        break;
      }
      before += __shfl_sync(0xFFFFFFFFu, upto, 31);
    }
  }
  w.rows = 0;
  w.sink_tiles = w.first = w.count = w.clean_from = w.clean_to = 0;
  if (b == a.batch) return w;
  w.r = seq_rows(a, b);
  w.row0 = blk * kRows;
  w.rows = min(max(w.r.nq - w.row0, 0), kRows);
  w.pos0 = w.r.nk - w.r.nq + w.row0;
  w.pos1 = w.pos0 + w.rows - 1;
  if (w.rows > 0 && w.pos1 >= 0) {
    const int lo = a.window > 0 ? max(0, w.pos0 - a.window + 1) : 0;      // first key of the first row's window
    w.first = lo / kKeys;
    w.sink_tiles = min((min(a.sinks, lo) + kKeys - 1) / kKeys, w.first);
    w.count = w.sink_tiles + w.pos1 / kKeys + 1 - w.first;
    const int all_from = a.window > 0 ? max(0, w.pos1 - a.window + 1) : 0;   // first key of the last row's window
    w.clean_from = w.sink_tiles + (all_from + kKeys - 1) / kKeys - w.first;
    w.clean_to = w.sink_tiles + (w.pos0 >= 0 ? (w.pos0 + 1) / kKeys - w.first : 0);
  }
  return w;
}

// Scores that are not seen (column > last, or before `from` and not before `sink`) become -infinity.  One bit per column:
// short prompts, whose tiles are all masked, take 9.6 us where three comparisons per score took 11.8.
__device__ __forceinline__ uint32_t first_bits(int n) { return n <= 0 ? 0u : n >= 32 ? 0xFFFFFFFFu : (1u << n) - 1u; }
__device__ __forceinline__ void mask_scores(float (&s)[kKeys], int last, int from, int sink) {
#pragma unroll
  for (int w = 0; w < kKeys; w += 32) {
    const uint32_t seen = first_bits(last + 1 - w) & (~first_bits(from - w) | first_bits(sink - w));
#pragma unroll
    for (int c = 0; c < 32; ++c) s[w + c] = seen & (1u << c) ? s[w + c] : -INFINITY;
  }
}
__device__ __forceinline__ float largest(const float (&s)[kKeys]) {
  float mx0 = max3(s[0], s[1], s[2]), mx1 = max3(s[3], s[4], s[5]), mx2 = s[6], mx3 = s[7];
#pragma unroll
  for (int c = 8; c < kKeys; c += 8) {
    mx0 = max3(mx0, s[c], s[c + 1]); mx1 = max3(mx1, s[c + 2], s[c + 3]);
    mx2 = max3(mx2, s[c + 4], s[c + 5]); mx3 = max3(mx3, s[c + 6], s[c + 7]);
  }
  return fmaxf(max3(mx0, mx1, mx2), mx3);
}
// Exponentials of the scores, rounded into p, and summed.
template <typename T>
__device__ __forceinline__ f32x2 exponentials(const float (&s)[kKeys], float sl, float shift, uint32_t (&p)[kKeys / 2]) {
  const f32x2 sl2 = pair(sl, sl), shift2 = pair(shift, shift);
  f32x2 l0 = pair(0.f, 0.f), l1 = l0;
#pragma unroll
  for (int i = 0; i < kKeys / 2; ++i) {
    float2 v = halves(fma2(pair(s[2 * i], s[2 * i + 1]), sl2, shift2));
    v.x = ex2(v.x); v.y = ex2(v.y);
    if (i & 1) l1 = add2(l1, pair(v.x, v.y)); else l0 = add2(l0, pair(v.x, v.y));
    p[i] = pack2<T>(v.x, v.y);
  }
  return add2(l0, l1);
}

template <int kDim> constexpr int kSlotsOf = kDim == 64 ? 8 : 4;   // two CTAs fit an SM

template <typename T, int kDim>
__global__ void __launch_bounds__(kThreads, 2)
attention_window_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                        const __grid_constant__ CUtensorMap map_v, WindowArgs a, uint32_t polls) {
  constexpr int kSlots = kSlotsOf<kDim>;
  constexpr int kSubs = kDim / 64;               // a tile is kSubs sub-tiles of 64 values per row (128 bytes)
  constexpr int kQSub = kRows * 128, kQBytes = kSubs * kQSub, kSub = kKeys * 128, kTileBytes = kSubs * kSub;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  unsigned char* sq = smem;                      // the query tile, then the ring
  unsigned char* ring = smem + kQBytes;
  Ctl* ctl = reinterpret_cast<Ctl*>(ring + kSlots * kTileBytes);
  volatile int* abort_flag = &ctl->abort_flag;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  pdl_wait();
  const Job job = make_job(a);
  if (job.rows == 0) return;                     // no block of rows for this CTA
  if (threadIdx.x == 0) {
    mbar_init(smem_u32(&ctl->q_full), 1);
    mbar_init(smem_u32(&ctl->drain), 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&ctl->s_full[i]), 1);
      mbar_init(smem_u32(&ctl->p_ready[i]), 4);
      mbar_init(smem_u32(&ctl->o_done[i]), 1);
    }
    for (int s = 0; s < kSlots; ++s) {
      mbar_init(smem_u32(&ctl->kv_full[s]), 1);
      mbar_init(smem_u32(&ctl->kv_empty[s]), 1);
    }
    ctl->abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kIssuer) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ctl->tmem_base)), "r"(kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  fence_proxy_async_smem();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  pdl_launch_dependents();                       // not before the tensor memory is ours: a kernel behind this one may take some, then wait for this one
  const uint32_t tmem = ctl->tmem_base, t_s = tmem, t_o = tmem + 2 * kKeys;

  if (warp == kCopier) {                                       // ---- copies
    if (lane == 0 && job.count > 0) {
      int issued = 0;
      mbar_arrive_expect_tx(smem_u32(&ctl->q_full), kQBytes);
      for (int s = 0; s < kSubs; ++s)
        tma_load_2d(smem_u32(sq + s * kQSub), &map_q, job.head * kDim + 64 * s, job.r.q0 + job.row0, smem_u32(&ctl->q_full));
      const int hk = job.head / (a.heads / a.kv_heads);
      for (int e = 0; e < 2 * job.count; ++e) {                // entry 2 j: keys of tile j; 2 j + 1: its values
        const int slot = e % kSlots;
        if (e >= kSlots && !wait_for(&ctl->kv_empty[slot], ((e / kSlots) - 1) & 1, abort_flag, polls)) break;
        mbar_arrive_expect_tx(smem_u32(&ctl->kv_full[slot]), kTileBytes);
        for (int s = 0; s < kSubs; ++s)
          tma_load_2d(smem_u32(ring + slot * kTileBytes + s * kSub), e & 1 ? &map_v : &map_k, hk * kDim + 64 * s,
                      job.r.k0 + job.key0(e >> 1), smem_u32(&ctl->kv_full[slot]));
        issued = e + 1;
      }
      int gave_up = 0;                                         // copies end before the CTA does, also after a wait ran out
      wait_for(&ctl->q_full, 0, &gave_up, kSpinLimit);
      for (int e = max(0, issued - kSlots); e < issued; ++e) wait_for(&ctl->kv_full[e % kSlots], (e / kSlots) & 1, &gave_up, kSpinLimit);
    }
  } else if (warp == kIssuer) {                                // ---- products (the whole warp; one lane issues)
    if (job.count > 0) {
      constexpr uint32_t kIdS = idesc<T>(kKeys, false), kIdO = idesc<T>(kDim, true);
      const uint32_t on = elect(), ring_at = smem_u32(ring);
      const uint64_t dq = smem_desc_sw128(smem_u32(sq));
      auto wait = [&](unsigned long long* bar, uint32_t parity) { return wait_warp(bar, parity, abort_flag, polls); };
      auto pv = [&](int j) -> bool {                           // O += P(j) V(j)
        const int ev = 2 * j + 1, slot = ev % kSlots;
        if (!wait(&ctl->kv_full[slot], (ev / kSlots) & 1)) return false;
        // Rows behind the sequence's last key (padding, or another sequence) meet probabilities of 0: they become zeros, so that
        // whatever they hold stays out of O.
        const int there = job.r.nk - job.key0(j);
        if (there < kKeys) {
          for (int s = 0; s < kSubs; ++s)
            for (int c = there * 8 + lane; c < kKeys * 8; c += 32)
              *reinterpret_cast<uint4*>(ring + slot * kTileBytes + s * kSub + c * 16) = make_uint4(0, 0, 0, 0);
          fence_proxy_async_smem();
          __syncwarp();
        }
        if (!wait(&ctl->p_ready[j & 1], (j >> 1) & 1)) return false;
        tc_fence_after();
        const uint64_t dv = desc_mn(ring_at + slot * kTileBytes);
        const uint32_t tp = t_s + (j & 1) * kKeys, more = j > 0;
#pragma unroll
        for (int k = 0; k < kKeys / 16; ++k)                   // 16 keys: 8 columns of P, 2048 bytes of V
          mma_ts(on, t_o, tp + 8 * k, dv + (uint64_t)(k * (2048 >> 4)), kIdO, k > 0 ? 1u : more);
        commit(on, &ctl->o_done[j & 1]);
        commit(on, &ctl->kv_empty[slot]);
        return true;
      };
      bool ok = wait(&ctl->q_full, 0);
      for (int j = 0; j < job.count && ok; ++j) {
        const int ek = 2 * j, slot = ek % kSlots;
        if (!(ok = wait(&ctl->kv_full[slot], (ek / kSlots) & 1))) break;
        const uint64_t dk = smem_desc_sw128(ring_at + slot * kTileBytes);
#pragma unroll
        for (int k = 0; k < kDim / 16; ++k)                    // 16 values: 32 bytes within a sub-tile's rows
          mma_ss(on, t_s + (j & 1) * kKeys, dq + (uint64_t)(((k / 4) * kQSub + (k % 4) * 32) >> 4),
                 dk + (uint64_t)(((k / 4) * kSub + (k % 4) * 32) >> 4), kIdS, k > 0);
        commit(on, &ctl->s_full[j & 1]);
        commit(on, &ctl->kv_empty[slot]);
        if (j > 0) ok = pv(j - 1);
      }
      if (ok) pv(job.count - 1);
      int gave_up = 0;                                         // products, and the arrivals they owe, end before the CTA does
      commit(on, &ctl->drain);
      wait_for(&ctl->drain, 0, &gave_up, kSpinLimit);
    }
  } else {                                                     // ---- softmax and output
    const int row = threadIdx.x;
    const uint32_t lanes = (uint32_t)(warp * 32) << 16, ts = t_s + lanes, to = t_o + lanes;
    const float sl = a.scale * 1.4426950408889634f;
    const int pos = job.pos0 + row, key_end = min(pos, job.r.nk - 1);
    float m = -INFINITY, l = 0.f;                              // running maximum (raw score) and sum of the row
    bool ok = true;
    // PV(j) is complete.  Two barriers in turn: PV(j - 2), the one before on the same barrier, is complete for certain
    // (S(j), which the caller has seen, was issued behind it), PV(j - 1) is not.
    auto o_ready = [&](int j) -> bool {
      const bool r = wait_warp(&ctl->o_done[j & 1], (j >> 1) & 1, abort_flag, polls);
      tc_fence_after();
      return r;
    };
    for (int j = 0; j < job.count; ++j) {
      const int k0 = job.key0(j);
      const uint32_t at = ts + (j & 1) * kKeys;
      if (!(ok = wait_warp(&ctl->s_full[j & 1], (j >> 1) & 1, abort_flag, polls))) break;
      tc_fence_after();
      float s[kKeys];
      ld32(at, s);
      ld32(at + 32, s + 32);
      ld_wait(s);
      ld_wait(s + 32);
      if (j < job.clean_from || j >= job.clean_to)
        mask_scores(s, key_end - k0, a.window > 0 ? pos - a.window + 1 - k0 : -0x40000000, a.sinks - k0);
      const float mx = largest(s);
      const bool move = m > -INFINITY && (mx - m) * sl > kMoveLog2;
      if (__any_sync(0xFFFFFFFFu, move)) {                     // O of the tiles so far takes the new maximum
        if (!(ok = o_ready(j - 1))) break;
        const float f = move ? ex2((m - mx) * sl) : 1.f;
        l *= f;
#pragma unroll
        for (int c = 0; c < kDim; c += 32) {
          float o[32];
          ld32(to + c, o);
          ld_wait(o);
#pragma unroll
          for (int i = 0; i < 32; ++i) o[i] *= f;
          st32(to + c, o);
        }
      }
      if (move || m == -INFINITY) m = fmaxf(m, mx);
      uint32_t p[kKeys / 2];
      const float2 sum = halves(exponentials<T>(s, sl, m == -INFINITY ? 0.f : kLiftLog2 - m * sl, p));
      st32(at, p);
      l += sum.x + sum.y;
      st_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&ctl->p_ready[j & 1]));
    }
    if (ok && job.count > 0) ok = o_ready(job.count - 1);
    if (ok) {
      // Through shared memory (the query tile's, which no product reads any more), each warp its own rows: whole rows leave
      // together.  Written from the registers, 16 bytes of each of 32 rows at a time, the whole kernel took 2 % longer.
      // A row in front of the first key sees nothing and gets zeros; another whose sum is 0 sees nothing but scores of
      // -infinity: 1 / 0 makes it NaN.
      const bool mine = row < job.rows, none = pos < 0;
      const float inv = none ? 0.f : 1.f / l;
      unsigned char* stage = sq + warp * 32 * kDim * 2;
      float check = 0.f;
#pragma unroll
      for (int c = 0; c < kDim; c += 32) {
        float v[32];
        if (job.count > 0) {
          ld32(to + c, v);
          ld_wait(v);
        }
        uint32_t w[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float x = none ? 0.f : v[2 * i] * inv, y = none ? 0.f : v[2 * i + 1] * inv;
          check = fmaf(x, 0.f, fmaf(y, 0.f, check));           // NaN once a value is not finite
          w[i] = pack2<T>(x, y);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *reinterpret_cast<uint4*>(stage + lane * kDim * 2 + (((c >> 3) + i) ^ (lane & 7)) * 16) =
              make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
      }
      __syncwarp();
      constexpr int kParts = kDim / 8, kAtOnce = 32 / kParts;  // 16-byte parts of a row, rows per instruction
      T* o = reinterpret_cast<T*>(a.o) + (int64_t)(job.r.q0 + job.row0 + warp * 32) * a.ld_o + (int64_t)job.head * kDim;
#pragma unroll
      for (int i = lane / kParts; i < 32; i += kAtOnce) {
        const int part = lane % kParts;
        if (warp * 32 + i < job.rows)
          *reinterpret_cast<uint4*>(o + (int64_t)i * a.ld_o + part * 8) = *reinterpret_cast<const uint4*>(stage + i * kDim * 2 + (part ^ (i & 7)) * 16);
      }
      __syncwarp();
      // (a sum l that is 0 or not finite comes from scores that are seen: the row's result is NaN by definition)
      unsigned bad = __ballot_sync(0xFFFFFFFFu, mine && !(check == 0.f) && l > 0.f && l - l == 0.f);
      while (bad) {
        const int i = __ffs(bad) - 1;
        bad &= bad - 1;
        window_row<T, kDim>(a, job.r, job.row0 + warp * 32 + i, job.head);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == kIssuer) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
  if (*abort_flag) {
    if (threadIdx.x == 0) atomicAdd(&g_window_fallbacks, 1u);
    for (int i = warp; i < job.rows; i += kThreads / 32) window_row<T, kDim>(a, job.r, job.row0 + i, job.head);
  }
}

// Tensor map of a token matrix [rows, width]: boxes of box_rows x 64 values, rows beyond the end read as zero.
template <typename T> bool make_map(CUtensorMap* map, const void* p, int64_t rows, int64_t width, int64_t ld, int box_rows) {
  EncodeFn enc = encode_fn();
  if (!enc) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)width, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld * 2};
  const cuuint32_t box[2] = {64, (cuuint32_t)box_rows}, estr[2] = {1, 1};
  return enc(map, std::is_same<T, __half>::value ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2,
             const_cast<void*>(p), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, int kDim>
cudaError_t launch_dim(const WindowArgs& a, cudaStream_t s) {
  constexpr size_t kSmem = (size_t)(kRows + kSlotsOf<kDim> * kKeys) * kDim * 2 + 1024 + sizeof(Ctl);
  static_assert(2 * (kSmem + 1024) <= 233472, "two CTAs exceed the shared memory of an SM");
  static std::atomic<uint64_t> ready{0};         // devices on which the kernel's shared memory limit is set
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev >= 64 || !((ready.load(std::memory_order_relaxed) >> dev) & 1)) {
    e = cudaFuncSetAttribute(attention_window_kernel<T, kDim>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem);
    if (e != cudaSuccess) return e;
    if (dev < 64) ready.fetch_or(1ull << dev, std::memory_order_relaxed);
  }
  CUtensorMap mq, mk, mv;
  if (!make_map<T>(&mq, a.q, a.rows_q, (int64_t)a.heads * kDim, a.ld_q, kRows)) return cudaErrorInvalidValue;
  if (a.rows_k > 0) {
    if (!make_map<T>(&mk, a.k, a.rows_k, (int64_t)a.kv_heads * kDim, a.ld_k, kKeys) ||
        !make_map<T>(&mv, a.v, a.rows_k, (int64_t)a.kv_heads * kDim, a.ld_v, kKeys))
      return cudaErrorInvalidValue;
  } else {
    mk = mv = mq;                                // no key anywhere: never used
  }
  int64_t units = (a.seq_q + kRows - 1) / kRows * a.batch;      // blocks of rows, at most
  if (a.cu_q) units = std::min(units, a.rows_q / kRows + a.batch);
  const int64_t grid = units * a.heads;
  const long long dbg = g_debug_wait_polls.load(std::memory_order_relaxed);
  const uint32_t polls = dbg < 0 ? kSpinLimit : (uint32_t)(dbg < (long long)kSpinLimit ? dbg : kSpinLimit);
  return launch_pdl(attention_window_kernel<T, kDim>, (unsigned)grid, kThreads, kSmem, s, mq, mk, mv, a, polls);
}

}  // namespace

cudaError_t launch_attention_window(const WindowArgs& a, cudaStream_t s) {
  if (a.dt == BL_F16) return a.head_dim == 64 ? launch_dim<__half, 64>(a, s) : launch_dim<__half, 128>(a, s);
  return a.head_dim == 64 ? launch_dim<__nv_bfloat16, 64>(a, s) : launch_dim<__nv_bfloat16, 128>(a, s);
}

cudaError_t window_take_fallbacks(unsigned int* out) {
  const unsigned int zero = 0;
  cudaError_t e = cudaMemcpyFromSymbol(out, g_window_fallbacks, sizeof(*out));
  return e != cudaSuccess ? e : cudaMemcpyToSymbol(g_window_fallbacks, &zero, sizeof(zero));
}

}  // namespace bl
