// Residual's addition, root-mean-square norm and 8-bit codes with a scale per token, in one pass:
//   h = residual + x   (or residual + sum_j p_j x[r_j]: the rows that a token's experts left, weighed)
//   y = w . h / sqrt(mean h^2 + eps),   scale = max |y| / 127,   code = round(y / scale).
// Bound by memory (and by instructions for the 16-bit types): x and the residual are read once, h and the codes written once, and a
// row stays in the registers of its threads in between.  The norm's factor is the same for the whole row and positive, so it cancels in the codes:
//   code = round(h w . 127 / max |h w|),   scale = max |h w| / (127 sqrt(mean h^2 + eps)),
// and one reduction that carries the sum of squares and the largest |h w| together serves both.
// Rows whose squares, or whose products with w, leave the range of fp32 go round again: once for the mean, scaled by the power of two
// that their largest value asks for, and once for the products, scaled by one that those ask for (a value that dwarfs the others may have
// a small weight).  They are loaded anew for it, a chunk of eight values at a time, so that this costs the others no registers.
#include <type_traits>

#include "common.cuh"

namespace bl {

namespace {

constexpr int kMaxWarps = 32;

// Eight consecutive values; loads are coherent, since outputs may be the inputs.
template <typename T> struct Eight { uint4 r; };
template <> struct Eight<float> { uint4 r, r2; };
template <typename T> __device__ __forceinline__ Eight<T> load_eight(const T* p) {
  Eight<T> v;
  v.r = *reinterpret_cast<const uint4*>(p);
  if constexpr (sizeof(T) == 4) v.r2 = *(reinterpret_cast<const uint4*>(p) + 1);
  return v;
}
// Values are held and worked on in pairs (packed fp32 arithmetic).
__device__ __forceinline__ float2 bits2(uint32_t a, uint32_t b) { return make_float2(__uint_as_float(a), __uint_as_float(b)); }
__device__ __forceinline__ void floats(const Eight<float>& e, float2 (&v)[4]) {
  v[0] = bits2(e.r.x, e.r.y); v[1] = bits2(e.r.z, e.r.w); v[2] = bits2(e.r2.x, e.r2.y); v[3] = bits2(e.r2.z, e.r2.w);
}
__device__ __forceinline__ void floats(const Eight<__half>& e, float2 (&v)[4]) {
  const __half2* h = reinterpret_cast<const __half2*>(&e.r);
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = __half22float2(h[i]);
}
__device__ __forceinline__ void floats(const Eight<__nv_bfloat16>& e, float2 (&v)[4]) {
  const uint32_t w[4] = {e.r.x, e.r.y, e.r.z, e.r.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = bits2(w[i] << 16, w[i] & 0xFFFF0000u);
}
__device__ __forceinline__ void store_eight(float* p, const float2 (&v)[4]) {
  *reinterpret_cast<float4*>(p) = make_float4(v[0].x, v[0].y, v[1].x, v[1].y);
  *reinterpret_cast<float4*>(p + 4) = make_float4(v[2].x, v[2].y, v[3].x, v[3].y);
}
__device__ __forceinline__ void store_eight(__half* p, const float2 (&v)[4]) {
  uint4 r;
  __half2* h = reinterpret_cast<__half2*>(&r);
#pragma unroll
  for (int i = 0; i < 4; ++i) h[i] = __float22half2_rn(v[i]);
  *reinterpret_cast<uint4*>(p) = r;
}
__device__ __forceinline__ void store_eight(__nv_bfloat16* p, const float2 (&v)[4]) {
  uint4 r;
  __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&r);
#pragma unroll
  for (int i = 0; i < 4; ++i) h[i] = __float22bfloat162_rn(v[i]);
  *reinterpret_cast<uint4*>(p) = r;
}
__device__ __forceinline__ float2 both(float f) { return make_float2(f, f); }
template <typename T> __device__ __forceinline__ void add_eight(float2 (&h)[4], const Eight<T>& v) {
  float2 f[4];
  floats(v, f);
#pragma unroll
  for (int e = 0; e < 4; ++e) h[e] = __fadd2_rn(h[e], f[e]);
}
template <typename T> __device__ __forceinline__ void add_eight(float2 (&h)[4], const Eight<T>& v, float p) {
  float2 f[4];
  floats(v, f);
#pragma unroll
  for (int e = 0; e < 4; ++e) h[e] = __ffma2_rn(both(p), f[e], h[e]);
}
// Eight ones, as stored.
template <typename T> __device__ __forceinline__ Eight<T> ones() {
  Eight<T> v;
  const uint32_t w = sizeof(T) == 4 ? 0x3F800000u : std::is_same<T, __half>::value ? 0x3C003C00u : 0x3F803F80u;
  v.r = make_uint4(w, w, w, w);
  if constexpr (sizeof(T) == 4) v.r2 = v.r;
  return v;
}
// The largest of one and the sizes of a pair; a NaN stays.
__device__ __forceinline__ float max_of(float a, float2 v) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(fabsf(v.x)), "f"(fabsf(v.y)));
  return r;
}
// max that keeps a NaN
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ bool finite(float f) { return (__float_as_uint(f) & 0x7F800000u) != 0x7F800000u; }

// The threads of a row: `warps` warps, of which there may be several groups in a block.  Sum and largest value over
// them, in a fixed order, the same bits in every thread.
struct RowThreads {
  float2* part;              // [2][warps], in turns so that one barrier per reduction is enough
  int warps, warp, lane, id, turn;
  __device__ RowThreads(float2* parts, int in_block, int i, int row_threads)
      : part(parts + in_block * 2 * (row_threads / 32)), warps(row_threads / 32), warp(i / 32), lane(i & 31), id(in_block + 1), turn(0) {}
  __device__ void sync() const {
    // Barriers by number as constants: with one in a register a block is taken to use all sixteen, and four blocks fit on an SM.  A
    // block has two groups of two warps, or one of any size.
    if (warps == 1) __syncwarp();
    else if (id == 1) asm volatile("bar.sync 1, %0;" ::"r"(warps * 32) : "memory");
    else asm volatile("bar.sync 2, %0;" ::"r"(warps * 32) : "memory");
  }
  __device__ void reduce(float& sum, float& top) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
      top = max_nan(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
    }
    if (warps == 1) return;
    float2* p = part + turn * warps;
    turn ^= 1;
    if (lane == 0) p[warp] = make_float2(sum, top);
    sync();
    float2 v = lane < warps ? p[lane] : make_float2(0.f, 0.f);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      v.x += __shfl_xor_sync(0xFFFFFFFFu, v.x, o);
      v.y = max_nan(v.y, __shfl_xor_sync(0xFFFFFFFFu, v.y, o));
    }
    sum = v.x; top = v.y;
  }
};

// What the outputs are made from: the products of values and weights times factor (y) and inv (codes).
struct RowResult { float factor, inv; bool fine; };

__device__ __forceinline__ float pow2(int n) { return __uint_as_float((uint32_t)(127 + n) << 23); }        // n in -126..127
__device__ __forceinline__ double pow2_wide(int n) { return __hiloint2double((1023 + n) << 20, 0); }       // n in -1022..1023
// v 2^n; what would pass fp32's largest stays there (scaled up, it belongs to a factor of 0 or to a product that is nothing beside the largest).
__device__ __forceinline__ void scale_eight(float2 (&v)[4], int n) {
  const float f = pow2(n), most = n > 0 ? 3.4028234e38f : INFINITY;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    v[e] = __fmul2_rn(v[e], both(f));
    if (n > 0) v[e] = make_float2(fminf(fmaxf(v[e].x, -most), most), fminf(fmaxf(v[e].y, -most), most));
  }
}

template <typename T>
__device__ __forceinline__ void store_products(const NormQuantArgs& a, int t, int at, const float2 (&p)[4], const RowResult& r) {
  if (a.y) {
    float2 v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = __fmul2_rn(p[e], both(r.factor));
    store_eight(reinterpret_cast<T*>(a.y) + (int64_t)t * a.ld_y + at * 8, v);
  }
  if (a.x_q) {
    // 1.5 2^23 + v has round(v), half to even, in its low bits; |v| <= 127 (1 + 2^-22) rounds into -127..127
    uint32_t q[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const float2 u = __ffma2_rn(p[2 * e], both(r.inv), both(12582912.f)), v = __ffma2_rn(p[2 * e + 1], both(r.inv), both(12582912.f));
      q[e] = __byte_perm(__byte_perm(__float_as_uint(u.x), __float_as_uint(u.y), 0x0040),
                         __byte_perm(__float_as_uint(v.x), __float_as_uint(v.y), 0x0040), 0x5410);
    }
    *reinterpret_cast<uint2*>(a.x_q + (int64_t)t * a.ld_q + at * 8) = r.fine ? make_uint2(q[0], q[1]) : make_uint2(0u, 0u);
  }
}
__device__ __forceinline__ RowResult result_of(const NormQuantArgs& a, int t, int i, float top, float factor) {
  RowResult r;
  r.fine = finite(top);
  r.factor = factor;
  r.inv = r.fine && top > 0.f ? 127.f / top : 0.f;
  if (a.x_q && i == 0) a.scale[t] = r.fine ? top * factor * (1.f / 127.f) : __uint_as_float(0x7FC00000u);
  return r;
}

// Squares or products out of fp32's range, or so small that they lost bits.
__device__ __forceinline__ bool out_of_range(float f) {          // below 1e-30 (of the positive), infinite or NaN
  return __float_as_uint(f) - 0x0DA24260u >= 0x7F800000u - 0x0DA24260u;
}

// Powers of two by which the values and the weights of a row whose products leave the range are multiplied, both, so that a product that
// counts has two factors in range: products that overflow are 2^128 to 2^256, those that are too small 2^-99 at most (in a second step
// those below 2^-250).  Scaled up, a factor that passes fp32's range had 2^53 (2^8) or more, and a partner of 0: as 2^-149 is the least.
constexpr int kDown = -65, kUp = 75, kFurtherUp = 120;

// The chunks of h (zeros behind the row).
template <typename T, int kChunks, bool kJoin>
__device__ __forceinline__ void fetch(const NormQuantArgs& a, int t, int i, int row_threads, int chunks, float2 (&h)[kChunks][4]) {
  const T* x = reinterpret_cast<const T*>(a.x);
  Eight<T> xs[kJoin ? 1 : kChunks];
#pragma unroll
  for (int c = 0; c < kChunks; ++c) {
    const int at = i + c * row_threads;
    Eight<T> r{};
    if constexpr (!kJoin) xs[c] = Eight<T>{};
    if (at < chunks) {
      if constexpr (!kJoin) xs[c] = load_eight(x + (int64_t)t * a.ld_x + at * 8);
      if (a.residual) r = load_eight(reinterpret_cast<const T*>(a.residual) + (int64_t)t * a.ld_res + at * 8);
    }
    floats(r, h[c]);
  }
  if constexpr (!kJoin) {
#pragma unroll
    for (int c = 0; c < kChunks; ++c) add_eight(h[c], xs[c]);
  } else {
    // Four rows at a time, all on their way together; one that is not there is a row of zeros with the weight 0.
    const int32_t* rows = a.rows + (int64_t)t * a.top_k;
    const float* shares = a.row_weights ? a.row_weights + (int64_t)t * a.top_k : nullptr;
#pragma unroll 1
    for (int j0 = 0; j0 < a.top_k; j0 += 4) {
      int32_t r[4];
      float p[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        r[j] = j0 + j < a.top_k ? rows[j0 + j] : -1;
        p[j] = shares && j0 + j < a.top_k ? shares[j0 + j] : 1.f;
        if (r[j] >= a.x_rows) r[j] = -1;
        if (r[j] < 0) p[j] = 0.f;
      }
#pragma unroll
      for (int c = 0; c < kChunks; ++c) {
        const int at = i + c * row_threads;
        Eight<T> v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          v[j] = Eight<T>{};
          if (at < chunks && r[j] >= 0) v[j] = load_eight(x + (int64_t)r[j] * a.ld_x + at * 8);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) add_eight(h[c], v[j], p[j]);
      }
    }
  }
}

template <typename T>
__device__ __forceinline__ Eight<T> load_weight(const NormQuantArgs& a, int at, int chunks) {
  return a.weight && a.eps >= 0.f && at < chunks ? load_eight(reinterpret_cast<const T*>(a.weight) + at * 8) : ones<T>();
}

// A row whose mean or whose largest product left the range; result is what the first round made of it.
template <typename T, bool kJoin>
__device__ __forceinline__ void far_row(const NormQuantArgs& a, int t, int i, int row_threads, int chunks, float top, RowResult result, RowThreads& rt) {
  const bool norm = a.eps >= 0.f;
  // its largest size, the mean of its squares scaled by 2^mean_scale, the largest product of values and weights scaled by 2^scale each
  // (once or twice), and its outputs from products scaled by 2^shift
  enum { kMost, kMean, kProducts, kLast };
  int round = kMost, mean_scale = 0, scale = !out_of_range(top) ? 0 : top < 1e-30f ? kUp : kDown, shift = 0;
  float root = 1.f;                                    // 1 / sqrt(mean of the scaled squares and eps)
#pragma unroll 1
  for (;;) {
    float sum = 0.f;
    top = 0.f;
#pragma unroll 1
    for (int at = i; at < chunks; at += row_threads) {
      float2 h[1][4], w[4];
      fetch<T, 1, kJoin>(a, t, at, row_threads, chunks, h);
      if (round == kLast && a.h) store_eight(reinterpret_cast<T*>(a.h) + (int64_t)t * a.ld_h + at * 8, h[0]);
      floats(round >= kProducts ? load_weight<T>(a, at, chunks) : ones<T>(), w);
      if (round == kMean) scale_eight(h[0], mean_scale);
      if (round >= kProducts && scale != 0) {
        scale_eight(h[0], scale);
        scale_eight(w, scale);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        sum = fmaf(h[0][e].x, h[0][e].x, fmaf(h[0][e].y, h[0][e].y, sum));
        w[e] = __fmul2_rn(h[0][e], w[e]);
        top = max_of(top, w[e]);
      }
      if (round == kLast) {
        if (shift != 0) {                              // up to 2^126 either way: in two steps
          scale_eight(w, shift / 2);
          scale_eight(w, shift - shift / 2);
        }
        store_products<T>(a, t, at, w, result);
      }
    }
    if (round == kLast) return;
    rt.reduce(sum, top);
    if (round == kMost) {
      if (top == 0.f) result.factor = 0.f;             // a row of zeros stays one, with eps = 0 too
      if (top == 0.f && a.x_q && i == 0 && result.fine) a.scale[t] = 0.f;
      if (top == 0.f || !finite(top)) scale = 0;
      // the largest goes to [1, 2) or [1, 4), or as near as a factor of 2^100 comes
      mean_scale = max(-126, min(100, 127 - max(1, (int)(__float_as_uint(top) >> 23))));
      round = top == 0.f || !finite(top) ? kLast : norm ? kMean : kProducts;
    } else if (round == kMean) {
      // 1 / sqrt(mean h^2 + eps) = f / sqrt(mean (f h)^2 + f^2 eps), f = 2^mean_scale; where f^2 eps passes fp32, the mean is nothing beside it
      const float f = pow2(mean_scale), scaled_eps = a.eps * f * f;
      root = finite(scaled_eps) ? rsqrtf(fmaf(sum, a.inv_k, scaled_eps)) : rsqrtf(a.eps);
      if (!finite(scaled_eps)) mean_scale = 0;
      round = kProducts;
    } else if (scale == kUp && top > 0.f && top < 7.8886091e-31f) {       // 2^-100
      scale = kFurtherUp;
    } else {
      // The products are brought to [1, 2) at their largest, and what is left of the powers of two goes into one factor: that of y is
      // about the largest y, and that of the codes 127 or less.  With a weight that is not finite the others' y are as they are.
      const bool apply = finite(top) && top > 0.f;
      if (!finite(top)) scale = 0;
      shift = apply ? 127 - max(1, (int)(__float_as_uint(top) >> 23)) : 0;
      const double factor = (double)root * pow2_wide((norm ? mean_scale : 0) - 2 * scale - shift);
      const float normal = apply ? top * pow2(shift / 2) * pow2(shift - shift / 2) : 0.f;
      result.fine = finite(top);
      result.factor = top == 0.f ? 0.f : (float)factor;
      result.inv = apply ? 127.f / normal : 0.f;
      if (a.x_q && i == 0) a.scale[t] = !result.fine ? __uint_as_float(0x7FC00000u) : (float)(factor * normal * (1. / 127.));
      round = kLast;
    }
  }
}

// Thread i of a row holds the chunks of eight values i, i + threads, ..., kChunks of them at most.
template <typename T, int kChunks, int kThreads, bool kJoin>
__global__ void __launch_bounds__(kThreads, kChunks == 2 ? 2 : 1) rms_norm_quant_kernel(NormQuantArgs a, int row_threads) {
  __shared__ float2 part[2 * kMaxWarps];
  pdl_launch_dependents();
  const int per_block = blockDim.x == row_threads ? 1 : blockDim.x / row_threads;
  const int in_block = per_block == 1 ? 0 : threadIdx.x / row_threads, i = threadIdx.x - in_block * row_threads;
  RowThreads rt(part, in_block, i, row_threads);
  const int t = (int)blockIdx.x * per_block + in_block;
  if (t >= (int)a.T) return;                              // whole rows of threads: none waits for another's
  pdl_wait();
  const int chunks = (int)(a.K / 8);
  const bool norm = a.eps >= 0.f;
  RowResult result{1.f, 0.f, true};
  float2 h[kChunks][4];
  {
    Eight<T> weight[kChunks];
#pragma unroll
    for (int c = 0; c < kChunks; ++c) weight[c] = load_weight<T>(a, i + c * row_threads, chunks);
    fetch<T, kChunks, kJoin>(a, t, i, row_threads, chunks, h);
    if (a.y || a.x_q) {
      // the sum of squares and the largest |h w|
      float2 s[2] = {both(0.f), both(0.f)};
      float m[2] = {0.f, 0.f};
#pragma unroll
      for (int c = 0; c < kChunks; ++c) {
        float2 w[4];
        floats(weight[c], w);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s[e & 1] = __ffma2_rn(h[c][e], h[c][e], s[e & 1]);
          m[e & 1] = max_of(m[e & 1], __fmul2_rn(h[c][e], w[e]));
        }
      }
      float sum = (s[0].x + s[0].y) + (s[1].x + s[1].y), top = max_nan(m[0], m[1]);
      rt.reduce(sum, top);
      const float mean = fmaf(sum, a.inv_k, a.eps);
      result = result_of(a, t, i, top, norm ? rsqrtf(mean) : 1.f);
      if (out_of_range(top) || (norm && out_of_range(mean))) {
        far_row<T, kJoin>(a, t, i, row_threads, chunks, top, result, rt);
        return;
      }
    }
  }
  if (a.h) {
    T* out = reinterpret_cast<T*>(a.h) + (int64_t)t * a.ld_h;
#pragma unroll
    for (int c = 0; c < kChunks; ++c)
      if (i + c * row_threads < chunks) store_eight(out + (i + c * row_threads) * 8, h[c]);
  }
#pragma unroll
  for (int c = 0; c < kChunks; ++c) {
    const int at = i + c * row_threads;
    if (at >= chunks) continue;
    float2 w[4];
    floats(load_weight<T>(a, at, chunks), w);             // again, from L1: registers are worth more
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = __fmul2_rn(w[e], h[c][e]);
    store_products<T>(a, t, at, w, result);
  }
}

template <typename T, int kChunks, int kThreads>
cudaError_t launch_chunks(const NormQuantArgs& a, int row_threads, cudaStream_t s) {
  const int per_block = row_threads >= 128 ? 1 : 128 / row_threads;
  const int64_t blocks = (a.T + per_block - 1) / per_block;
  const auto kern = a.rows ? rms_norm_quant_kernel<T, kChunks, kThreads, true> : rms_norm_quant_kernel<T, kChunks, kThreads, false>;
  return launch_pdl(kern, (unsigned)blocks, (unsigned)(row_threads * per_block), 0, s, a, row_threads);
}

template <typename T>
cudaError_t launch_type(const NormQuantArgs& a, cudaStream_t s) {
  const int chunks = (int)(a.K / 8);
  auto threads = [&](int per) { return ((chunks + per - 1) / per + 31) / 32 * 32; };
  // Up to a row per SM: as many threads as there are chunks (1 x 4096: 2.0 us, with two chunks a thread 2.1, with four 2.5).  More: two
  // chunks a thread share what every thread does once per row (8191 x 4096 fp32: one chunk 90 us, two 66, four 67; bf16: 67, 42.8, 40.7;
  // 149 x 8192 bf16 4.8, 3.6, 3.7).
  if (threads(1) <= 64 || (a.T <= 148 && threads(1) <= 1024)) return launch_chunks<T, 1, 1024>(a, threads(1), s);
  if (threads(2) <= 512) return launch_chunks<T, 2, 512>(a, threads(2), s);
  if (threads(4) <= 512) return launch_chunks<T, 4, 512>(a, threads(4), s);
  return launch_chunks<T, 4, 1024>(a, threads(4), s);
}

}  // namespace

cudaError_t launch_rms_norm_quant(const NormQuantArgs& a, cudaStream_t s) {
  switch (a.dt) {
    case BL_F32: return launch_type<float>(a, s);
    case BL_F16: return launch_type<__half>(a, s);
    default: return launch_type<__nv_bfloat16>(a, s);
  }
}

}  // namespace bl
