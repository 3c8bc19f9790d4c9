// The 4-bit key/value cache: quantising token rows into it, reading them back, copying its pages.
//   eta = min x, step = (max x - min x) / 15 (rounded to the cache's type), code = clip(rint((x - eta) / step)).
// All three are bound by memory.  Append and read give each (token, head) row kDim / 16 lanes, 16 values per
// lane in two runs of 8, half a row apart (a warp's access then covers whole sectors): two 16-byte accesses to the 16-bit
// rows, 2 x 4 bytes of key codes and two words of value codes.
#include <type_traits>

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
template <typename T> __device__ __forceinline__ uint32_t bits_of(float v) {
  const T x = out_cast<T>(v);
  return *reinterpret_cast<const uint16_t*>(&x);
}
template <typename T> __device__ __forceinline__ uint32_t nan_pair();
template <> __device__ __forceinline__ uint32_t nan_pair<__half>() { return 0x7E007E00u; }
template <> __device__ __forceinline__ uint32_t nan_pair<__nv_bfloat16>() { return 0x7FC07FC0u; }

// The code of a value whose quotient (x - eta) / step is within one of the code c, in exact arithmetic: in fp64 x - eta and
// code * step are exact, so the residual against half a step decides, ties to the even code.
__device__ __forceinline__ uint32_t border_code(float x, float eta, float step, int c) {
  const double d = (double)x - (double)eta, s = (double)step, r = fma(-(double)c, s, d), h = 0.5 * s;
  if (r > h || (r == h && (c & 1))) ++c;
  else if (r < -h || (r == -h && (c & 1))) --c;
  return (uint32_t)min(max(c, 0), 15);
}
// The same from any quotient (steps so small or so large that fp32 does not serve).
__device__ __noinline__ uint32_t exact_code(float x, float eta, float step) {
  if (!(step > 0.f)) return 0;
  const double q = rint(((double)x - (double)eta) / (double)step);
  return border_code(x, eta, step, (int)fmin(fmax(q, 0.0), 16.0));
}
// RN_T((hi - lo) / 15).  The fp32 quotient is within 2^-22 of the exact one; where rounding it 2^-21 lower and higher
// gives two results, fp64 decides.
template <typename T> __device__ __noinline__ uint32_t step_bits64(float lo, float hi) { return round_bits<T>(((double)hi - (double)lo) / 15.0); }
template <typename T> __device__ __forceinline__ uint32_t step_bits(float lo, float hi) {
  const float q = (hi - lo) * (1.0f / 15.0f);
  const uint32_t down = bits_of<T>(q * (1.f - 0x1p-21f)), up = bits_of<T>(q * (1.f + 0x1p-21f));
  return down == up && q < 1e38f ? down : step_bits64<T>(lo, hi);
}
// Smaller of two pairs, each half for itself; a NaN wins.
template <typename T> __device__ __forceinline__ uint32_t min_pairs(uint32_t a, uint32_t b);
template <> __device__ __forceinline__ uint32_t min_pairs<__half>(uint32_t a, uint32_t b) {
  const __half2 m = __hmin2_nan(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
  return *reinterpret_cast<const uint32_t*>(&m);
}
template <> __device__ __forceinline__ uint32_t min_pairs<__nv_bfloat16>(uint32_t a, uint32_t b) {
  const __nv_bfloat162 m = __hmin2_nan(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
  return *reinterpret_cast<const uint32_t*>(&m);
}

// A row's 16 codes of this lane as nibbles (value i in bits 4 i % 32 of word i / 8), and the row's (step, eta) word.
// In fp32 the quotient (x - eta) / step is off by less than 4e-6 (it is at most 15 and a bit, and three roundings enter),
// so a value whose quotient lies further than 1e-5 from a border between codes has its code from the fp32 sum with
// 1.5 * 2^23, whose low bits are the rounded quotient.  Others go to fp64: with bf16 rows about one value in 300 lies on a
// border exactly, so that path is short.  Steps below the type's normal range (quotients may pass 15.5) or at the end of
// fp32's take exact_code.
template <typename T, int kLanes>
__device__ __forceinline__ void quantise_row(const uint4 (&raw)[2], uint32_t (&nib)[2], uint32_t& scale) {
  constexpr float kMagic = 12582912.f;
  constexpr float kLeast = std::is_same<T, __half>::value ? 6.2e-5f : 1e-30f;
  const uint32_t w[8] = {raw[0].x, raw[0].y, raw[0].z, raw[0].w, raw[1].x, raw[1].y, raw[1].z, raw[1].w};
  // smallest value and smallest negated value, side by side in one word through the shuffles
  uint32_t mn = w[0], mx = w[0] ^ 0x80008000u;
#pragma unroll
  for (int i = 1; i < 8; ++i) { mn = min_pairs<T>(mn, w[i]); mx = min_pairs<T>(mx, w[i] ^ 0x80008000u); }
  uint32_t both = min_pairs<T>(__byte_perm(mn, mx, 0x5410), __byte_perm(mn, mx, 0x7632));
#pragma unroll
  for (int o = kLanes / 2; o > 0; o >>= 1) both = min_pairs<T>(both, __shfl_xor_sync(0xFFFFFFFFu, both, o));
  const float2 ends = scale_floats<T>(both);
  const float lo = ends.x, hi = -ends.y;
  const uint32_t sb = step_bits<T>(lo, hi);
  const float step = scale_floats<T>(sb).x;
  float inv;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(step));
  uint32_t doubt = 0;                                 // values whose quotient is too near a border, one bit each
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    float c[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float2 f = scale_floats<T>(w[4 * k + i / 2]);
      const float d = (i & 1 ? f.y : f.x) - lo;
      c[i] = fmaf(d, inv, kMagic) - kMagic;
      if (fabsf(fmaf(d, inv, -c[i])) > 0.49999f) doubt |= 1u << (8 * k + i);
    }
    const float n0 = fmaf(c[1], 16.f, c[0]) + fmaf(c[3], 4096.f, c[2] * 256.f);
    const float n1 = fmaf(c[5], 16.f, c[4]) + fmaf(c[7], 4096.f, c[6] * 256.f);
    nib[k] = __byte_perm(__float_as_uint(n0 + 8388608.f), __float_as_uint(n1 + 8388608.f), 0x5410);
  }
  const bool odd_step = !(step > kLeast && step < 1e30f);
  if (odd_step) doubt = 0xFFFFu;
  if (step == 0.f) { nib[0] = nib[1] = 0; doubt = 0; }   // a constant row (or no row at all)
#pragma unroll 1
  while (doubt) {
    const int i = __ffs(doubt) - 1, shift = 4 * (i & 7);
    doubt &= doubt - 1;
    const uint32_t a0 = i & 2 ? w[1] : w[0], a1 = i & 2 ? w[3] : w[2], a2 = i & 2 ? w[5] : w[4], a3 = i & 2 ? w[7] : w[6];
    const uint32_t b0 = i & 4 ? a1 : a0, b1 = i & 4 ? a3 : a2, have = i & 8 ? nib[1] : nib[0];
    const float2 f = scale_floats<T>(i & 8 ? b1 : b0);
    const float x = i & 1 ? f.y : f.x;
    const uint32_t code = odd_step ? exact_code(x, lo, step) : border_code(x, lo, step, (int)((have >> shift) & 15u));
    const uint32_t made = (have & ~(15u << shift)) | (code << shift);
    if (i & 8) nib[1] = made; else nib[0] = made;
  }
  scale = __byte_perm(sb, both, 0x5410);
  if (!(lo >= -3.4e38f && hi <= 3.4e38f)) { nib[0] = nib[1] = 0; scale = nan_pair<T>(); }
}

// Where a lane's part of a (token, head) row lies; kUnroll rows per lane, a block's rows interleaved.
struct Place { char* block; int j; bool on; };
template <int kDim> __device__ __forceinline__ Place place_of(const bl_kv4_cache& c, int64_t slot, int h) {
  const int pl = 31 - __clz(c.page_size);             // page sizes are powers of two
  Place p;
  p.on = slot >= 0 && (slot >> pl) < c.num_pages;
  p.j = (int)slot & (c.page_size - 1);
  p.block = reinterpret_cast<char*>(c.pages) + ((slot >> pl) * c.kv_heads + h) * (int64_t)Block<kDim>::bytes(c.page_size);
  return p;
}
// The rows of a warp: 32 / kLanes consecutive tokens of one head (so that two tokens whose value codes interleave are
// neighbours), kUnroll times over.  job counts (run of tokens, head).
template <int kLanes, int kUnroll> struct Rows {
  uint32_t t0; int h;
  __device__ __forceinline__ Rows(int kv_heads) {
    const uint32_t job = blockIdx.x * (kKvThreads / 32) + (threadIdx.x >> 5), run = job / (uint32_t)kv_heads;
    h = (int)(job - run * (uint32_t)kv_heads);
    t0 = run * (32 / kLanes * kUnroll) + (threadIdx.x & 31) / kLanes;
  }
  __device__ __forceinline__ int64_t token(int u) const { return (int64_t)t0 + u * (32 / kLanes); }
};

template <typename T, int kDim, int kUnroll>
__global__ void __launch_bounds__(kKvThreads, 4) kv4_append_kernel(bl_kv4_cache c, const T* __restrict__ k, const T* __restrict__ v,
                                                               int64_t T_, int64_t ld_k, int64_t ld_v,
                                                               const int64_t* __restrict__ slots) {
  constexpr int kLanes = kDim / 16;
  const int lane = threadIdx.x & 31, sub = lane % kLanes, d0 = sub * 8, d1 = kDim / 2 + d0, odd = (lane / kLanes) & 1;
  const Rows<kLanes, kUnroll> rows(c.kv_heads);
  pdl_launch_dependents();
  pdl_wait();
  uint4 kr[kUnroll][2], vr[kUnroll][2];
  int64_t slot[kUnroll];
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    const int64_t t = rows.token(u);
    slot[u] = t < T_ ? slots[t] : -1;
    kr[u][0] = kr[u][1] = vr[u][0] = vr[u][1] = make_uint4(0, 0, 0, 0);
    if (t < T_) {
      const T* kp = k + t * ld_k + (int64_t)rows.h * kDim;
      const T* vp = v + t * ld_v + (int64_t)rows.h * kDim;
      kr[u][0] = __ldg(reinterpret_cast<const uint4*>(kp + d0)); kr[u][1] = __ldg(reinterpret_cast<const uint4*>(kp + d1));
      vr[u][0] = __ldg(reinterpret_cast<const uint4*>(vp + d0)); vr[u][1] = __ldg(reinterpret_cast<const uint4*>(vp + d1));
    }
  }
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    uint32_t kn[2], ks, vn[2], vs;
    quantise_row<T, kLanes>(kr[u], kn, ks);
    quantise_row<T, kLanes>(vr[u], vn, vs);
    const Place p = place_of<kDim>(c, slot[u], rows.h);
    // two tokens in neighbouring slots share words of value codes: each lane of the pair writes two whole words
    const int64_t other = __shfl_xor_sync(0xFFFFFFFFu, slot[u], kLanes);
    const uint32_t theirs = __shfl_xor_sync(0xFFFFFFFFu, odd ? vn[0] : vn[1], kLanes);
    if (!p.on) continue;
    *reinterpret_cast<uint32_t*>(p.block + p.j * (kDim / 2) + d0 / 2) = kn[0];
    *reinterpret_cast<uint32_t*>(p.block + p.j * (kDim / 2) + d1 / 2) = kn[1];
    char* vc = p.block + Block<kDim>::v_codes(c.page_size);
    if ((slot[u] ^ other) == 1 && (p.j & 1) == odd) {
      const uint32_t lo = odd ? theirs : vn[0], hi = odd ? vn[1] : theirs;
      *reinterpret_cast<uint2*>(vc + Block<kDim>::v_at(p.j & ~1, odd ? d1 : d0)) = make_uint2(__byte_perm(lo, hi, 0x5410), __byte_perm(lo, hi, 0x7632));
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<uint16_t*>(vc + Block<kDim>::v_at(p.j, (i < 2 ? d0 : d1) + 4 * (i & 1))) = (uint16_t)(vn[i >> 1] >> (16 * (i & 1)));
    }
    if (sub == 0) *reinterpret_cast<uint32_t*>(p.block + Block<kDim>::k_scale(c.page_size) + 4 * p.j) = ks;
    if (sub == 1) *reinterpret_cast<uint32_t*>(p.block + Block<kDim>::v_scale(c.page_size) + 4 * p.j) = vs;
  }
}

// eta + step * code of two neighbouring codes, as stored; 2^23 + code is the float with the code in its low bits.
template <typename T> __device__ __forceinline__ uint32_t two_values(uint32_t nib, int at, float2 se) {
  const float c0 = __uint_as_float(0x4B000000u | ((nib >> at) & 15u)) - 8388608.f;
  const float c1 = __uint_as_float(0x4B000000u | ((nib >> (at + 4)) & 15u)) - 8388608.f;
  const T a = out_cast<T>(fmaf(c0, se.x, se.y)), b = out_cast<T>(fmaf(c1, se.x, se.y));
  return (uint32_t)*reinterpret_cast<const uint16_t*>(&a) | ((uint32_t)*reinterpret_cast<const uint16_t*>(&b) << 16);
}
template <typename T> __device__ __forceinline__ void store_values(T* p, uint32_t nib, float2 se) {
  *reinterpret_cast<uint4*>(p) = make_uint4(two_values<T>(nib, 0, se), two_values<T>(nib, 8, se), two_values<T>(nib, 16, se), two_values<T>(nib, 24, se));
}

template <typename T, int kDim, int kUnroll>
__global__ void __launch_bounds__(kKvThreads) kv4_read_kernel(bl_kv4_cache c, T* __restrict__ k, T* __restrict__ v, int64_t T_,
                                                             int64_t ld_k, int64_t ld_v, const int64_t* __restrict__ slots) {
  constexpr int kLanes = kDim / 16;
  const int d0 = ((threadIdx.x & 31) % kLanes) * 8, d1 = kDim / 2 + d0;
  const Rows<kLanes, kUnroll> rows(c.kv_heads);
  pdl_launch_dependents();
  pdl_wait();
  uint2 kn[kUnroll], v0[kUnroll], v1[kUnroll];         // key codes; words of value codes, of this token and its pair's other
  uint32_t ks[kUnroll], vs[kUnroll];
  bool on[kUnroll], high[kUnroll];
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    const int64_t t = rows.token(u);
    const Place p = place_of<kDim>(c, t < T_ ? __ldg(slots + t) : -1, rows.h);
    on[u] = p.on;
    high[u] = p.j & 1;
    kn[u] = v0[u] = v1[u] = make_uint2(0, 0);
    ks[u] = vs[u] = 0;
    if (p.on) {
      const char* vc = p.block + Block<kDim>::v_codes(c.page_size);
      kn[u].x = *reinterpret_cast<const uint32_t*>(p.block + p.j * (kDim / 2) + d0 / 2);
      kn[u].y = *reinterpret_cast<const uint32_t*>(p.block + p.j * (kDim / 2) + d1 / 2);
      v0[u] = *reinterpret_cast<const uint2*>(vc + Block<kDim>::v_at(p.j & ~1, d0));
      v1[u] = *reinterpret_cast<const uint2*>(vc + Block<kDim>::v_at(p.j & ~1, d1));
      ks[u] = *reinterpret_cast<const uint32_t*>(p.block + Block<kDim>::k_scale(c.page_size) + 4 * p.j);
      vs[u] = *reinterpret_cast<const uint32_t*>(p.block + Block<kDim>::v_scale(c.page_size) + 4 * p.j);
    }
  }
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    if (!on[u]) continue;
    const int64_t t = rows.token(u);
    T* kp = k + t * ld_k + (int64_t)rows.h * kDim;
    T* vp = v + t * ld_v + (int64_t)rows.h * kDim;
    const float2 kse = scale_floats<T>(ks[u]), vse = scale_floats<T>(vs[u]);
    const uint32_t pick = high[u] ? 0x7632u : 0x5410u;
    store_values<T>(kp + d0, kn[u].x, kse); store_values<T>(kp + d1, kn[u].y, kse);
    store_values<T>(vp + d0, __byte_perm(v0[u].x, v0[u].y, pick), vse); store_values<T>(vp + d1, __byte_perm(v1[u].x, v1[u].y, pick), vse);
  }
}

// One CTA copies kCopyBytes of one page of one layer; 16 bytes per access, all loads of a thread in flight at once.
constexpr int kCopyUnroll = 8;
constexpr int kCopyBytes = kKvThreads * 16 * kCopyUnroll;

__global__ void __launch_bounds__(kKvThreads) kv4_copy_kernel(char* pages, int64_t page_bytes, int64_t num_pages, int64_t layer_stride,
                                                             const int2* __restrict__ pairs, unsigned chunks) {
  pdl_launch_dependents();
  pdl_wait();
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

// Rows per lane: kMany where that still fills the GPU eight times over, so that a lane has that many loads in flight; else one.
constexpr int kMany = 2;
unsigned row_blocks(const bl_kv4_cache& c, int64_t T, int unroll) {
  const int64_t run = 32 / (c.head_dim / 16) * unroll, jobs = (T + run - 1) / run * c.kv_heads;
  return (unsigned)((jobs + kKvThreads / 32 - 1) / (kKvThreads / 32));
}

template <typename T, int kDim>
cudaError_t append_dim(const bl_kv4_cache& c, const void* k, const void* v, int64_t n, int64_t ld_k, int64_t ld_v,
                       const int64_t* slots, cudaStream_t s) {
  const T* kp = reinterpret_cast<const T*>(k);
  const T* vp = reinterpret_cast<const T*>(v);
  const unsigned many = row_blocks(c, n, kMany);
  if (many >= 8 * 148) return launch_pdl(kv4_append_kernel<T, kDim, kMany>, many, kKvThreads, 0, s, c, kp, vp, n, ld_k, ld_v, slots);
  return launch_pdl(kv4_append_kernel<T, kDim, 1>, row_blocks(c, n, 1), kKvThreads, 0, s, c, kp, vp, n, ld_k, ld_v, slots);
}
template <typename T>
cudaError_t append_type(const bl_kv4_cache& c, const void* k, const void* v, int64_t n, int64_t ld_k, int64_t ld_v,
                        const int64_t* slots, cudaStream_t s) {
  return c.head_dim == 64 ? append_dim<T, 64>(c, k, v, n, ld_k, ld_v, slots, s) : append_dim<T, 128>(c, k, v, n, ld_k, ld_v, slots, s);
}

template <typename T, int kDim>
cudaError_t read_dim(const bl_kv4_cache& c, void* k, void* v, int64_t n, int64_t ld_k, int64_t ld_v, const int64_t* slots,
                     cudaStream_t s) {
  T* kp = reinterpret_cast<T*>(k);
  T* vp = reinterpret_cast<T*>(v);
  const unsigned many = row_blocks(c, n, kMany);
  if (many >= 8 * 148) return launch_pdl(kv4_read_kernel<T, kDim, kMany>, many, kKvThreads, 0, s, c, kp, vp, n, ld_k, ld_v, slots);
  return launch_pdl(kv4_read_kernel<T, kDim, 1>, row_blocks(c, n, 1), kKvThreads, 0, s, c, kp, vp, n, ld_k, ld_v, slots);
}
template <typename T>
cudaError_t read_type(const bl_kv4_cache& c, void* k, void* v, int64_t n, int64_t ld_k, int64_t ld_v, const int64_t* slots,
                      cudaStream_t s) {
  return c.head_dim == 64 ? read_dim<T, 64>(c, k, v, n, ld_k, ld_v, slots, s) : read_dim<T, 128>(c, k, v, n, ld_k, ld_v, slots, s);
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
  return launch_pdl(kv4_copy_kernel, dim3((unsigned)n * chunks, (unsigned)layers), kKvThreads, 0, s, reinterpret_cast<char*>(pages),
                    (int64_t)page_bytes, num_pages, (int64_t)layer_stride, reinterpret_cast<const int2*>(pairs), chunks);
}

}  // namespace bl
