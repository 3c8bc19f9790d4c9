// The 4-bit key/value cache: quantising token rows into it, reading them back, copying its pages.
//   eta = min x, step = (max x - min x) / 15 (rounded to the cache's type), code = clip(rint((x - eta) / step)).
// All three are bound by memory.  Append and read give each (token, head) row kDim / 8 lanes, 8 values per
// lane: one 16-byte access to the 16-bit rows, 4 bytes of key codes and 2 x 2 bytes of value codes.
#include "kv4.cuh"

namespace bl {

namespace {

using namespace kv4;

constexpr int kKvThreads = 256;

template <typename T> __device__ __forceinline__ uint32_t round_bits(double v);
template <> __device__ __forceinline__ uint32_t round_bits<__half>(double v) { return __half_as_ushort(__double2half(v)); }
template <> __device__ __forceinline__ uint32_t round_bits<__nv_bfloat16>(double v) {
  return __bfloat16_as_ushort(__double2bfloat16(v));
}
template <typename T> __device__ __forceinline__ uint32_t nan_pair();
template <> __device__ __forceinline__ uint32_t nan_pair<__half>() { return 0x7E007E00u; }
template <> __device__ __forceinline__ uint32_t nan_pair<__nv_bfloat16>() { return 0x7FC07FC0u; }

// rint((x - eta) / step) decided as in exact arithmetic.  In fp32 the quotient is off by less than 4e-6 (its
// size is at most 15 and a bit, three roundings), so only quotients within 1e-5 of a border go to fp64, where
// x - eta and code * step are exact: the residual against half a step then decides, ties to the even code.
__device__ __forceinline__ uint32_t code_of(float x, float eta, float step, float inv) {
  const float f = (x - eta) * inv;
  float c = rintf(f);
  if (!(fabsf(f - c) <= 0.49999f)) {                  // near a border; and when f is not finite
    const double d = (double)x - (double)eta, s = (double)step;
    double e = s > 0.0 ? rint(d / s) : 0.0;
    e = fmin(fmax(e, 0.0), 16.0);
    const double r = fma(-e, s, d), h = 0.5 * s;
    if (r > h || (r == h && ((int)e & 1))) e += 1.0;
    else if (r < -h || (r == -h && ((int)e & 1))) e -= 1.0;
    c = s > 0.0 ? (float)e : 0.f;
  }
  return (uint32_t)(int)fminf(fmaxf(c, 0.f), 15.f);
}

// A row's 8 codes of this lane as nibbles (value i in bits 4 i), and the row's (step, eta) word.
template <typename T, int kLanes>
__device__ __forceinline__ void quantise_row(const float (&v)[8], uint32_t& nib, uint32_t& scale) {
  float lo = v[0], hi = v[0], sum = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) { lo = fminf(lo, v[i]); hi = fmaxf(hi, v[i]); sum += v[i] * 0.f; }   // sum: NaN unless all finite
#pragma unroll
  for (int o = kLanes / 2; o > 0; o >>= 1) {
    lo = fminf(lo, __shfl_xor_sync(0xFFFFFFFFu, lo, o));
    hi = fmaxf(hi, __shfl_xor_sync(0xFFFFFFFFu, hi, o));
    sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
  }
  const uint32_t sb = round_bits<T>(((double)hi - (double)lo) / 15.0);
  const float step = scale_floats<T>(sb).x;
  // steps at the ends of the fp32 range go to the fp64 path: their reciprocal is not accurate, or not finite
  const float inv = step > 1e-30f && step < 1e30f ? 1.0f / step : __int_as_float(0x7FC00000);
  nib = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) nib |= code_of(v[i], lo, step, inv) << (4 * i);
  scale = sb | (round_bits<T>((double)lo) << 16);     // lo is a value of T: nothing is rounded
  if (!(sum == 0.f)) { nib = 0; scale = nan_pair<T>(); }
}

template <typename T, int kDim>
__global__ void __launch_bounds__(kKvThreads) kv4_append_kernel(bl_kv4_cache c, const T* __restrict__ k, const T* __restrict__ v,
                                                               int64_t T_, int64_t ld_k, int64_t ld_v,
                                                               const int64_t* __restrict__ slots) {
  constexpr int kLanes = kDim / 8, kRows = kKvThreads / kLanes;
  const int sub = threadIdx.x % kLanes, d = sub * 8;
  const int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / kLanes;
  const int64_t t = row / c.kv_heads;
  const int h = (int)(row % c.kv_heads);
  const int64_t slot = t < T_ ? slots[t] : -1;
  const bool on = slot >= 0 && slot < c.num_pages * (int64_t)c.page_size;
  float kx[8] = {}, vx[8] = {};
  if (on) {
    Elem<T>::load8(k + t * ld_k + (int64_t)h * kDim + d, kx);
    Elem<T>::load8(v + t * ld_v + (int64_t)h * kDim + d, vx);
  }
  uint32_t kn, ks, vn, vs;
  quantise_row<T, kLanes>(kx, kn, ks);
  quantise_row<T, kLanes>(vx, vn, vs);
  if (!on) return;
  const int j = (int)(slot % c.page_size);
  char* block = reinterpret_cast<char*>(c.pages) + ((slot / c.page_size) * c.kv_heads + h) * (int64_t)Block<kDim>::bytes(c.page_size);
  *reinterpret_cast<uint32_t*>(block + j * (kDim / 2) + d / 2) = kn;
  char* vc = block + Block<kDim>::v_codes(c.page_size);
  *reinterpret_cast<uint16_t*>(vc + Block<kDim>::v_at(j, d)) = (uint16_t)vn;
  *reinterpret_cast<uint16_t*>(vc + Block<kDim>::v_at(j, d + 4)) = (uint16_t)(vn >> 16);
  if (sub == 0) *reinterpret_cast<uint32_t*>(block + Block<kDim>::k_scale(c.page_size) + 4 * j) = ks;
  if (sub == 1) *reinterpret_cast<uint32_t*>(block + Block<kDim>::v_scale(c.page_size) + 4 * j) = vs;
}

template <typename T> __device__ __forceinline__ void store_values(T* p, uint32_t nib, float2 se);
template <> __device__ __forceinline__ void store_values<__half>(__half* p, uint32_t nib, float2 se) {
  uint4 r;
  __half2* o = reinterpret_cast<__half2*>(&r);
#pragma unroll
  for (int i = 0; i < 4; ++i)
    o[i] = __floats2half2_rn(fmaf((float)((nib >> (8 * i)) & 15u), se.x, se.y), fmaf((float)((nib >> (8 * i + 4)) & 15u), se.x, se.y));
  *reinterpret_cast<uint4*>(p) = r;
}
template <> __device__ __forceinline__ void store_values<__nv_bfloat16>(__nv_bfloat16* p, uint32_t nib, float2 se) {
  uint4 r;
  __nv_bfloat162* o = reinterpret_cast<__nv_bfloat162*>(&r);
#pragma unroll
  for (int i = 0; i < 4; ++i)
    o[i] = __floats2bfloat162_rn(fmaf((float)((nib >> (8 * i)) & 15u), se.x, se.y), fmaf((float)((nib >> (8 * i + 4)) & 15u), se.x, se.y));
  *reinterpret_cast<uint4*>(p) = r;
}

template <typename T, int kDim>
__global__ void __launch_bounds__(kKvThreads) kv4_read_kernel(bl_kv4_cache c, T* __restrict__ k, T* __restrict__ v, int64_t T_,
                                                             int64_t ld_k, int64_t ld_v, const int64_t* __restrict__ slots) {
  constexpr int kLanes = kDim / 8, kRows = kKvThreads / kLanes;
  const int d = (threadIdx.x % kLanes) * 8;
  const int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / kLanes;
  const int64_t t = row / c.kv_heads;
  const int h = (int)(row % c.kv_heads);
  if (t >= T_) return;
  const int64_t slot = slots[t];
  if (slot < 0 || slot >= c.num_pages * (int64_t)c.page_size) return;
  const int j = (int)(slot % c.page_size);
  const char* block = reinterpret_cast<const char*>(c.pages) +
                      ((slot / c.page_size) * c.kv_heads + h) * (int64_t)Block<kDim>::bytes(c.page_size);
  const char* vc = block + Block<kDim>::v_codes(c.page_size);
  const uint32_t kn = *reinterpret_cast<const uint32_t*>(block + j * (kDim / 2) + d / 2);
  const uint32_t vn = *reinterpret_cast<const uint16_t*>(vc + Block<kDim>::v_at(j, d)) |
                      ((uint32_t)*reinterpret_cast<const uint16_t*>(vc + Block<kDim>::v_at(j, d + 4)) << 16);
  const uint32_t ks = *reinterpret_cast<const uint32_t*>(block + Block<kDim>::k_scale(c.page_size) + 4 * j);
  const uint32_t vs = *reinterpret_cast<const uint32_t*>(block + Block<kDim>::v_scale(c.page_size) + 4 * j);
  store_values<T>(k + t * ld_k + (int64_t)h * kDim + d, kn, scale_floats<T>(ks));
  store_values<T>(v + t * ld_v + (int64_t)h * kDim + d, vn, scale_floats<T>(vs));
}

// One CTA copies kCopyBytes of one page of one layer; 16 bytes per access, all loads of a thread in flight at once.
constexpr int kCopyUnroll = 8;
constexpr int kCopyBytes = kKvThreads * 16 * kCopyUnroll;

__global__ void __launch_bounds__(kKvThreads) kv4_copy_kernel(char* pages, int64_t page_bytes, int64_t num_pages, int64_t layer_stride,
                                                             const int2* __restrict__ pairs, unsigned chunks) {
  const int2 pr = pairs[blockIdx.x / chunks];
  if (pr.x < 0 || pr.y < 0 || pr.x >= num_pages || pr.y >= num_pages || pr.x == pr.y) return;
  char* layer = pages + (int64_t)blockIdx.y * layer_stride;
  const int64_t off = (int64_t)(blockIdx.x % chunks) * kCopyBytes + threadIdx.x * 16;
  const char* src = layer + pr.x * page_bytes + off;
  char* dst = layer + pr.y * page_bytes + off;
  uint4 r[kCopyUnroll];
#pragma unroll
  for (int i = 0; i < kCopyUnroll; ++i)
    if (off + i * (kKvThreads * 16) < page_bytes) r[i] = *reinterpret_cast<const uint4*>(src + i * (kKvThreads * 16));
#pragma unroll
  for (int i = 0; i < kCopyUnroll; ++i)
    if (off + i * (kKvThreads * 16) < page_bytes) *reinterpret_cast<uint4*>(dst + i * (kKvThreads * 16)) = r[i];
}

unsigned row_blocks(const bl_kv4_cache& c, int64_t T) {
  const int rows = kKvThreads / (c.head_dim / 8);
  return (unsigned)((T * c.kv_heads + rows - 1) / rows);
}

template <typename T>
cudaError_t append_type(const bl_kv4_cache& c, const void* k, const void* v, int64_t n, int64_t ld_k, int64_t ld_v,
                        const int64_t* slots, cudaStream_t s) {
  const T* kp = reinterpret_cast<const T*>(k);
  const T* vp = reinterpret_cast<const T*>(v);
  if (c.head_dim == 64) kv4_append_kernel<T, 64><<<row_blocks(c, n), kKvThreads, 0, s>>>(c, kp, vp, n, ld_k, ld_v, slots);
  else kv4_append_kernel<T, 128><<<row_blocks(c, n), kKvThreads, 0, s>>>(c, kp, vp, n, ld_k, ld_v, slots);
  return cudaGetLastError();
}

template <typename T>
cudaError_t read_type(const bl_kv4_cache& c, void* k, void* v, int64_t n, int64_t ld_k, int64_t ld_v, const int64_t* slots,
                      cudaStream_t s) {
  T* kp = reinterpret_cast<T*>(k);
  T* vp = reinterpret_cast<T*>(v);
  if (c.head_dim == 64) kv4_read_kernel<T, 64><<<row_blocks(c, n), kKvThreads, 0, s>>>(c, kp, vp, n, ld_k, ld_v, slots);
  else kv4_read_kernel<T, 128><<<row_blocks(c, n), kKvThreads, 0, s>>>(c, kp, vp, n, ld_k, ld_v, slots);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_kv4_append(const bl_kv4_cache& c, const void* k, const void* v, int64_t T, int64_t ld_k, int64_t ld_v,
                              const int64_t* slots, cudaStream_t s) {
  return c.dtype == BL_F16 ? append_type<__half>(c, k, v, T, ld_k, ld_v, slots, s)
                           : append_type<__nv_bfloat16>(c, k, v, T, ld_k, ld_v, slots, s);
}

cudaError_t launch_kv4_read(const bl_kv4_cache& c, void* k, void* v, int64_t T, int64_t ld_k, int64_t ld_v,
                            const int64_t* slots, cudaStream_t s) {
  return c.dtype == BL_F16 ? read_type<__half>(c, k, v, T, ld_k, ld_v, slots, s)
                           : read_type<__nv_bfloat16>(c, k, v, T, ld_k, ld_v, slots, s);
}

cudaError_t launch_kv4_copy_pages(void* pages, size_t page_bytes, int64_t num_pages, int layers, size_t layer_stride,
                                  const int32_t* pairs, int64_t n, cudaStream_t s) {
  const unsigned chunks = (unsigned)((page_bytes + kCopyBytes - 1) / kCopyBytes);
  kv4_copy_kernel<<<dim3((unsigned)n * chunks, (unsigned)layers), kKvThreads, 0, s>>>(
      reinterpret_cast<char*>(pages), (int64_t)page_bytes, num_pages, (int64_t)layer_stride, reinterpret_cast<const int2*>(pairs),
      chunks);
  return cudaGetLastError();
}

}  // namespace bl
