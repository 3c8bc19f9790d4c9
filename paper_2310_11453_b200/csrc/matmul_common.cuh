// What the two kernels behind bitlinear_matmul_i8 and bitlinear_matmul_grouped share: the tensor-core instructions for
// both kinds of operands, the search for the rows of a tile, and what happens to a sum on its way out.
//
// Both compute the product transposed: the weights are the A operand (output features on the lanes of tensor memory), the
// tokens the B operand (columns).  So a token's outputs lie along the lanes of a warp, each store of a warp is one
// run of y, a feature's scale and bias are one register, and a list of rows may end anywhere without a tile of 128 tokens
// going to waste: the token tile is the narrow side of the instruction.
#pragma once

#include "tc_common.cuh"

namespace bl {
namespace mm {

using namespace tc;

constexpr int kRowBytes = 128;             // bytes of K per stage and row: one swizzle atom
constexpr int kMaxExperts = 1024;

// Instruction descriptor: both operands K-major; s8 x s8 -> s32, or fp16 / bf16 -> fp32.
__host__ __device__ constexpr uint32_t instr_desc(int operand, int m, int n) {
  return (operand == BL_I8 ? (2u << 4) | (1u << 7) | (1u << 10)
                           : (1u << 4) | (operand == BL_BF16 ? (1u << 7) | (1u << 10) : 0u)) |
         ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}

template <bool kInt, int kCtas>
__device__ __forceinline__ void mma(uint32_t d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
#define BL_MMA(CTAS, KIND)                                                                                  \
  asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\n"                                                  \
               "tcgen05.mma.cta_group::" CTAS ".kind::" KIND " [%0], %1, %2, %3, p;\n}" ::"r"(d), "l"(adesc), \
               "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory")
  if constexpr (kInt && kCtas == 1) BL_MMA("1", "i8");
  if constexpr (kInt && kCtas == 2) BL_MMA("2", "i8");
  if constexpr (!kInt && kCtas == 1) BL_MMA("1", "f16");
  if constexpr (!kInt && kCtas == 2) BL_MMA("2", "f16");
#undef BL_MMA
}

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int c0, int c1, int c2, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
      ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(bar) : "memory");
}
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* map, int c0, int c1, int c2, int c3, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
      ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(bar) : "memory");
}
// Brings a box into L2 and nowhere else.  Whoever writes there later writes to L2 as well: a hint, whatever the order of things.
__device__ __forceinline__ void tma_prefetch_4d(const CUtensorMap* map, int c0, int c1, int c2, int c3) {
  asm volatile("cp.async.bulk.prefetch.tensor.4d.L2.global [%0, {%1, %2, %3, %4}];" ::"l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(c3) : "memory");
}
__device__ __forceinline__ void st_cluster(uint32_t addr, uint32_t v) {
  asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}
__device__ __forceinline__ uint32_t ld_cluster(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.shared::cluster.b32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}
// Four rows of the matrix, wherever they lie, one under the other.
__device__ __forceinline__ void tma_gather4(uint32_t dst, const CUtensorMap* map, int c0, const int (&r)[4], uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile::gather4.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];"
      ::"r"(dst), "l"(map), "r"(c0), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(bar) : "memory");
}
// The same for a pair of CTAs: the bytes are counted on a barrier that may be the partner's (the copy lands in this CTA).
__device__ __forceinline__ void tma_load_2d_pair(uint32_t dst, const CUtensorMap* map, int c0, int c1, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
      ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(bar) : "memory");
}
__device__ __forceinline__ void tma_load_4d_pair(uint32_t dst, const CUtensorMap* map, int c0, int c1, int c2, int c3, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
      ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(bar) : "memory");
}
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
// Address of the same variable in CTA `rank` of this cluster.
__device__ __forceinline__ uint32_t map_to_rank(uint32_t local, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(local), "r"(rank));
  return r;
}
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void mbar_arrive_expect_tx_cluster(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cluster.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void mma_commit_pair(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void cluster_sync_all() {
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void prefetch_map(const CUtensorMap* map) {
  asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}

__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr));
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}

// offsets[e], cut to the list [0, R).
__device__ __forceinline__ int offset_of(const int32_t* offsets, int e, int R) {
  const int v = offsets[e];
  return v < 0 ? 0 : v > R ? R : v;
}

// The tiles of a launch, in the order in which every role of every CTA takes them: expert by expert, within one all row tiles of a
// feature tile first, so that CTAs that run at once share its weights.  The plan lies in shared memory: per expert the first row
// tile (and behind the last their number), the first row, the number of rows.
inline size_t plan_bytes(int experts) { return (size_t)(3 * experts + 1) * sizeof(int); }

// One warp makes the plan.  An offset below one before it counts as that one: whatever they are, the lists do not overlap, and there are no
// more tiles than the host reckoned with.
__device__ inline void make_plan(const MatmulArgs& a, int* plan, int tile_rows) {
  const int lane = threadIdx.x & 31;
  int *first = plan, *start = plan + a.experts + 1, *count = plan + 2 * a.experts + 1;
  int seen = 0, reached = 0;                 // tiles and rows of the experts before
  for (int base = 0; base < a.experts; base += 32) {
    const int e = base + lane;
    int from = 0, n = 0;
    if (a.offsets) {
      from = e < a.experts ? offset_of(a.offsets, e, (int)a.R) : 0;
      int to = e < a.experts ? offset_of(a.offsets, e + 1, (int)a.R) : 0;
      from = max(from, reached);
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xFFFFFFFFu, from, o);
        if (lane >= o) from = max(from, v);
      }
      to = max(to, from);
      n = to - from;
      reached = __shfl_sync(0xFFFFFFFFu, to, 31);
    } else if (e == 0) {
      n = (int)a.R;
    }
    if (e < a.experts) {
      start[e] = from;
      count[e] = n;
    } else {
      n = 0;
    }
    const int tiles = (n + tile_rows - 1) / tile_rows;
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

struct Walk {
  const int *first, *start, *count;
  uint32_t t, total, stride, feature_tiles;
  int e, row0, rows, f;                    // of the tile: expert, first row, rows, feature tile
  __device__ Walk(const int* plan, int experts, int feature_tiles_, uint32_t from, uint32_t stride_)
      : first(plan), start(plan + experts + 1), count(plan + 2 * experts + 1), t(from), total((uint32_t)plan[experts] * (uint32_t)feature_tiles_),
        stride(stride_), feature_tiles((uint32_t)feature_tiles_), e(0), row0(0), rows(0), f(0) {}
  __device__ bool valid() const { return t < total; }
  __device__ void next() { t += stride; }
  // An expert's rows are shared out evenly over its tiles, in multiples of `unit` rows.
  __device__ void locate(int unit) {
    while (t >= feature_tiles * (uint32_t)first[e + 1]) ++e;
    const uint32_t local = t - feature_tiles * (uint32_t)first[e], n = (uint32_t)(first[e + 1] - first[e]);
    f = (int)(local / n);
    const int each = (int)(((uint32_t)count[e] + n - 1) / n + unit - 1) / unit * unit, skip = (int)(local - (uint32_t)f * n) * each;
    row0 = start[e] + skip;
    rows = min(each, count[e] - skip);
  }
};

// The row of x behind a row of the list; one that does not exist reads as the nearest that does.
__device__ __forceinline__ int source_row(const MatmulArgs& a, int row) {
  const int r = a.rows ? a.rows[row] : row;
  return r < 0 ? 0 : r >= (int)a.x_rows ? (int)a.x_rows - 1 : r;
}

template <bool kInt> __device__ __forceinline__ float sum_value(uint32_t bits) {
  return kInt ? (float)(int32_t)bits : __uint_as_float(bits);
}

// Loads that stay where they are written, all on their way before the first is used.
template <typename TY> struct RawOf { using type = uint16_t; };
template <> struct RawOf<float> { using type = uint32_t; };
template <typename TY> using Raw = typename RawOf<TY>::type;
__device__ __forceinline__ uint32_t load_raw(const float* p) {
  uint32_t v;
  asm volatile("ld.global.b32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
  return v;
}
template <typename TY> __device__ __forceinline__ uint16_t load_raw(const TY* p) {
  uint16_t v;
  asm volatile("ld.global.b16 %0, [%1];" : "=h"(v) : "l"(p) : "memory");
  return v;
}
template <typename TY> __device__ __forceinline__ float raw_value(Raw<TY> v) { return in_cast(*reinterpret_cast<const TY*>(&v)); }

// What a feature's outputs have in common.
template <typename TY>
struct Feature {
  float scale, bias, least;                // least: 0 with a ReLU
  bool on;
  __device__ Feature(const MatmulArgs& a, int expert, int n) : scale(1.f), bias(0.f), least(a.relu ? 0.f : -INFINITY), on(n < a.N) {
    if (!on) return;
    const int64_t at = (int64_t)expert * a.N + n;
    if (a.w_scale) scale = a.w_scale[at];
    if (a.bias) bias = in_cast(reinterpret_cast<const TY*>(a.bias)[at]);
  }
  // (sum sx) sw + bias, of two rows: the product of the factors alone may leave fp32's range.  A NaN stays one through the ReLU.
  __device__ void finish2(float sum0, float sum1, float sx0, float sx1, float& v0, float& v1) const {
    const float2 v = __ffma2_rn(__fmul2_rn(make_float2(sum0, sum1), make_float2(sx0, sx1)), make_float2(scale, scale), make_float2(bias, bias));
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(v0) : "f"(v.x), "f"(least));
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(v1) : "f"(v.y), "f"(least));
  }
};

inline cudaError_t encode_rows(CUtensorMap* map, const void* base, int64_t row_bytes, int64_t rows, int64_t stride_bytes, int box_rows) {
  EncodeFn enc = encode_fn();
  if (!enc) return cudaErrorNotSupported;
  const cuuint64_t dims[2] = {(cuuint64_t)row_bytes, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)stride_bytes};
  const cuuint32_t box[2] = {(cuuint32_t)kRowBytes, (cuuint32_t)box_rows};
  const cuuint32_t estr[2] = {1, 1};
  return enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
             CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
             ? cudaSuccess : cudaErrorInvalidValue;
}
// A matrix (of several experts, if experts > 0) as boxes of box_rows x 128 bytes: of `sub` consecutive blocks of K at once, which
// lie behind each other in shared memory (sub > 0: K has to be a whole number of blocks), or of one at any byte of K (sub = 0).
// Coordinates: byte, row, block, expert.
inline cudaError_t encode_blocks(CUtensorMap* map, const void* base, int64_t row_bytes, int64_t rows, int64_t stride_bytes, int experts,
                                 int64_t expert_bytes, int box_rows, int sub) {
  EncodeFn enc = encode_fn();
  if (!enc) return cudaErrorNotSupported;
  const cuuint64_t dims[4] = {(cuuint64_t)(sub > 0 ? kRowBytes : row_bytes), (cuuint64_t)rows, (cuuint64_t)(sub > 0 ? row_bytes / kRowBytes : 1),
                              (cuuint64_t)(experts > 0 ? experts : 1)};
  const cuuint64_t strides[3] = {(cuuint64_t)stride_bytes, (cuuint64_t)kRowBytes, (cuuint64_t)(experts > 1 ? expert_bytes : stride_bytes)};
  const cuuint32_t box[4] = {(cuuint32_t)kRowBytes, (cuuint32_t)box_rows, (cuuint32_t)(sub > 0 ? sub : 1), 1};
  const cuuint32_t estr[4] = {1, 1, 1, 1};
  return enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, experts > 0 ? 4 : 3, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
             CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
             ? cudaSuccess : cudaErrorInvalidValue;
}

}  // namespace mm
}  // namespace bl
