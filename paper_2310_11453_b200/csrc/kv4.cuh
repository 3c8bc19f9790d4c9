// Layout of the 4-bit key/value cache (bl_kv4_cache in bitlinear.h), shared by the kernels that write,
// read and attend over it.
#pragma once

#include "common.cuh"

namespace bl {
namespace kv4 {

// Bytes of one head in a page, and where its parts start.
template <int kDim> struct Block {
  static __host__ __device__ __forceinline__ int bytes(int page_size) { return page_size * (kDim + 8); }
  static __host__ __device__ __forceinline__ int k_codes(int) { return 0; }
  static __host__ __device__ __forceinline__ int v_codes(int page_size) { return page_size * (kDim / 2); }
  static __host__ __device__ __forceinline__ int k_scale(int page_size) { return page_size * kDim; }
  static __host__ __device__ __forceinline__ int v_scale(int page_size) { return page_size * (kDim + 4); }
  // byte of value code d (d % 4 == 0: two bytes hold d..d+3) of token t, within the value codes
  static __host__ __device__ __forceinline__ int v_at(int t, int d) {
    const int e = d % (kDim / 8);
    return (t >> 3) * (4 * kDim) + ((d / (kDim / 8)) * 4 + ((t & 7) >> 1)) * (kDim / 8) + (e >> 2) * 4 + (t & 1) * 2;
  }
};

// How many parts a list of attention_kv4 has, of the slot (two per warp) of its first part and the warp of its last; 0 where
// the two do not name parts of `warps` warps (a workspace that nobody wrote may hold any bits).
__host__ __device__ inline int part_count(int first_slot, int last_warp, int warps) {
  const int w0 = first_slot >> 1;
  return w0 < 0 || last_warp < w0 || last_warp >= warps ? 0 : last_warp - w0 + 1;
}

// (step, eta) as stored: two 16-bit numbers of the cache's type.
template <typename T> __device__ __forceinline__ float2 scale_floats(uint32_t w);
template <> __device__ __forceinline__ float2 scale_floats<__half>(uint32_t w) {
  return __half22float2(*reinterpret_cast<const __half2*>(&w));
}
template <> __device__ __forceinline__ float2 scale_floats<__nv_bfloat16>(uint32_t w) {
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}

}  // namespace kv4
}  // namespace bl
