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

// A wait with a limit: 0 polls for a limit of 0.
__device__ __forceinline__ bool wait_for(uint32_t bar, uint32_t parity, volatile int* abort_flag, long long polls) {
  if (polls < 0) return mbar_wait(bar, parity, abort_flag);
  for (long long i = 0; i < polls; ++i) {
    if (mbar_try_wait(bar, parity)) return true;
    if (*abort_flag) return false;
  }
  *abort_flag = 1;
  return false;
}

// Waits for something that is sure to come (its own copies and products), whether or not others gave up; bounded all the same.
__device__ __forceinline__ void wait_quiet(uint32_t bar, uint32_t parity) {
  const unsigned long long t0 = global_ns();
  while (!mbar_try_wait(bar, parity))
    if (global_ns() - t0 > kWaitNs) return;
}

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
__device__ __forceinline__ void tma_load_3d_pair(uint32_t dst, const CUtensorMap* map, int c0, int c1, int c2, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
      ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(bar) : "memory");
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

// Rows of the list [0, R) that belong to expert e, from offsets that may be anything.
__device__ __forceinline__ int offset_of(const int32_t* offsets, int e, int R) {
  const int v = offsets[e];
  return v < 0 ? 0 : v > R ? R : v;
}

struct Tile { int expert, row0, rows; };   // rows: 0 where there is no such tile

// The i-th tile of up to kTile rows in the order of the experts.  All lanes of a warp call it.
__device__ inline Tile find_tile(const MatmulArgs& a, int i, int tile_rows) {
  Tile t{0, i * tile_rows, 0};
  if (!a.offsets) {
    const int64_t left = a.R - (int64_t)i * tile_rows;
    t.rows = left < 0 ? 0 : left > tile_rows ? tile_rows : (int)left;
    return t;
  }
  const int lane = threadIdx.x & 31;
  int seen = 0;
  for (int base = 0; base < a.experts; base += 32) {
    const int e = base + lane;
    int from = 0, n = 0;
    if (e < a.experts) {
      from = offset_of(a.offsets, e, (int)a.R);
      n = max(0, offset_of(a.offsets, e + 1, (int)a.R) - from);
    }
    const int tiles = (n + tile_rows - 1) / tile_rows;
    int upto = tiles;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xFFFFFFFFu, upto, o);
      if (lane >= o) upto += v;
    }
    const uint32_t hit = __ballot_sync(0xFFFFFFFFu, seen + upto > i);
    if (hit) {
      const int l = __ffs(hit) - 1;
      const int before = seen + upto - tiles;
      const int r0 = (i - before) * tile_rows;
      t.expert = base + l;
      t.row0 = __shfl_sync(0xFFFFFFFFu, from + r0, l);
      t.rows = __shfl_sync(0xFFFFFFFFu, min(tile_rows, n - r0), l);
      return t;
    }
    seen += __shfl_sync(0xFFFFFFFFu, upto, 31);
  }
  return t;
}

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
  float scale, bias;
  bool on;
  __device__ Feature(const MatmulArgs& a, int expert, int n) : scale(1.f), bias(0.f), on(n < a.N) {
    if (!on) return;
    const int64_t at = (int64_t)expert * a.N + n;
    if (a.w_scale) scale = a.w_scale[at];
    if (a.bias) bias = in_cast(reinterpret_cast<const TY*>(a.bias)[at]);
  }
  // (sum sx) sw: the factors alone may leave fp32's range.  A NaN stays one through the ReLU.
  __device__ float finish(const MatmulArgs& a, float sum, float x_scale) const {
    float v = sum * x_scale * scale + bias;
    if (a.relu) v = v < 0.f ? 0.f : v;
    return v;
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
inline cudaError_t encode_weights(CUtensorMap* map, const MatmulArgs& a, int box_rows) {
  EncodeFn enc = encode_fn();
  if (!enc) return cudaErrorNotSupported;
  const int es = a.operand == BL_I8 ? 1 : 2;
  const cuuint64_t dims[3] = {(cuuint64_t)(a.K * es), (cuuint64_t)a.N, (cuuint64_t)a.experts};
  const cuuint64_t strides[2] = {(cuuint64_t)(a.ld_w * es), (cuuint64_t)((a.experts > 1 ? a.expert_stride : a.ld_w) * es)};
  const cuuint32_t box[3] = {(cuuint32_t)kRowBytes, (cuuint32_t)box_rows, 1};
  const cuuint32_t estr[3] = {1, 1, 1};
  return enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<void*>(a.w), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
             CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
             ? cudaSuccess : cudaErrorInvalidValue;
}

}  // namespace mm
}  // namespace bl
