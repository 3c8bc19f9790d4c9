// Residual's addition, root-mean-square norm and 8-bit codes with a scale per token, in one pass:
//   h = residual + x   (or residual + sum_j p_j x[r_j]: the rows that a token's experts left, weighed)
//   y = w . h / sqrt(mean h^2 + eps),   scale = max |y| / 127,   code = round(y / scale).
// Bound by memory: x and the residual are read once, h and the codes written once, and a row stays in the registers of
// its threads in between.  The norm's factor is the same for the whole row and positive, so it cancels in the codes:
//   code = round(h w . 127 / max |h w|),   scale = max |h w| / (127 sqrt(mean h^2 + eps)),
// and one reduction that carries the sum of squares and the largest |h w| together serves both.
// Rows whose squares, or whose products with w, leave the range of fp32 go through a second pair of reductions over
// values scaled by a power of two (exact).
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
__device__ __forceinline__ void floats(const Eight<float>& e, float (&v)[8]) {
  v[0] = __uint_as_float(e.r.x); v[1] = __uint_as_float(e.r.y); v[2] = __uint_as_float(e.r.z); v[3] = __uint_as_float(e.r.w);
  v[4] = __uint_as_float(e.r2.x); v[5] = __uint_as_float(e.r2.y); v[6] = __uint_as_float(e.r2.z); v[7] = __uint_as_float(e.r2.w);
}
__device__ __forceinline__ void floats(const Eight<__half>& e, float (&v)[8]) {
  const __half2* h = reinterpret_cast<const __half2*>(&e.r);
#pragma unroll
  for (int i = 0; i < 4; ++i) { const float2 f = __half22float2(h[i]); v[2 * i] = f.x; v[2 * i + 1] = f.y; }
}
__device__ __forceinline__ void floats(const Eight<__nv_bfloat16>& e, float (&v)[8]) {
  const uint32_t w[4] = {e.r.x, e.r.y, e.r.z, e.r.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
}
__device__ __forceinline__ void store_eight(float* p, const float (&v)[8]) {
  *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void store_eight(__half* p, const float (&v)[8]) {
  uint4 r;
  __half2* h = reinterpret_cast<__half2*>(&r);
#pragma unroll
  for (int i = 0; i < 4; ++i) h[i] = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
  *reinterpret_cast<uint4*>(p) = r;
}
__device__ __forceinline__ void store_eight(__nv_bfloat16* p, const float (&v)[8]) {
  uint4 r;
  __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&r);
#pragma unroll
  for (int i = 0; i < 4; ++i) h[i] = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
  *reinterpret_cast<uint4*>(p) = r;
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
  __device__ void sync() const {
    if (warps == 1) __syncwarp();
    else asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(warps * 32) : "memory");
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

// Thread i of a row holds the chunks of eight values i, i + threads, ..., kChunks of them at most.
template <typename T, int kChunks, bool kJoin>
__global__ void __launch_bounds__(1024) rms_norm_quant_kernel(NormQuantArgs a, int row_threads) {
  __shared__ float2 part[2 * kMaxWarps];
  // Weights are quantised without the norm, and bitlinear_matmul_i8 reads weights ahead of the stream's order: what follows then starts
  // when these are written.
  if (a.eps >= 0.f) pdl_launch_dependents();
  const int in_block = threadIdx.x / row_threads, i = threadIdx.x - in_block * row_threads;
  RowThreads rt;
  rt.warps = row_threads / 32; rt.warp = i / 32; rt.lane = i & 31; rt.id = in_block + 1; rt.turn = 0;
  rt.part = part + in_block * 2 * rt.warps;
  const int64_t t = (int64_t)blockIdx.x * (blockDim.x / row_threads) + in_block;
  if (t >= a.T) return;                              // whole rows of threads: none waits for another's
  pdl_wait();
  const int chunks = (int)(a.K / 8);
  const bool norm = a.eps >= 0.f;
  const T* x = reinterpret_cast<const T*>(a.x);
  const T* res = a.residual ? reinterpret_cast<const T*>(a.residual) + t * a.ld_res : nullptr;
  const T* weight = norm ? reinterpret_cast<const T*>(a.weight) : nullptr;

  float h[kChunks][8];
  if constexpr (kJoin) {
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
      const int at = i + c * row_threads;
#pragma unroll
      for (int e = 0; e < 8; ++e) h[c][e] = 0.f;
      if (at < chunks && res) floats(load_eight(res + at * 8), h[c]);
    }
    const int32_t* rows = a.rows + t * a.top_k;
    const float* shares = a.row_weights ? a.row_weights + t * a.top_k : nullptr;
#pragma unroll 4
    for (int j = 0; j < a.top_k; ++j) {
      const int32_t r = rows[j];
      if (r < 0 || r >= a.x_rows) continue;          // no row: nothing is added
      const float p = shares ? shares[j] : 1.f;
#pragma unroll
      for (int c = 0; c < kChunks; ++c) {
        const int at = i + c * row_threads;
        if (at < chunks) {
          float v[8];
          floats(load_eight(x + (int64_t)r * a.ld_x + at * 8), v);
#pragma unroll
          for (int e = 0; e < 8; ++e) h[c][e] = fmaf(p, v[e], h[c][e]);
        }
      }
    }
  } else {
    Eight<T> xs[kChunks], rs[kChunks];
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
      const int at = i + c * row_threads;
      if (at < chunks) {
        xs[c] = load_eight(x + t * a.ld_x + at * 8);
        if (res) rs[c] = load_eight(res + at * 8);
      }
    }
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
      const int at = i + c * row_threads;
#pragma unroll
      for (int e = 0; e < 8; ++e) h[c][e] = 0.f;
      if (at < chunks) {
        floats(xs[c], h[c]);
        if (res) {
          float v[8];
          floats(rs[c], v);
#pragma unroll
          for (int e = 0; e < 8; ++e) h[c][e] += v[e];
        }
      }
    }
  }
  if (a.h) {
    T* out = reinterpret_cast<T*>(a.h) + t * a.ld_h;
#pragma unroll
    for (int c = 0; c < kChunks; ++c)
      if (i + c * row_threads < chunks) store_eight(out + (i + c * row_threads) * 8, h[c]);
  }
  if (!a.y && !a.x_q) return;

  // The sum of squares and the largest |h w|.  The products are formed again for the outputs: the weights come from L1, and
  // the registers serve more rows in flight.
  float sum = 0.f, top = 0.f;
  auto weights = [&](int at, float (&w)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = 1.f;
    if (weight) floats(load_eight(weight + at * 8), w);
  };
  auto measure = [&]() {
    sum = 0.f; top = 0.f;
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
      const int at = i + c * row_threads;
      if (at < chunks) {
        float w[8];
        weights(at, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          sum = fmaf(h[c][e], h[c][e], sum);
          top = max_nan(top, fabsf(h[c][e] * w[e]));
        }
      }
    }
    rt.reduce(sum, top);
  };
  measure();
  const float inv_k = 1.f / (float)a.K;
  float factor = norm ? rsqrtf(fmaf(sum, inv_k, a.eps)) : 1.f;
  bool divide = false;                               // codes by division rather than by 127 / top
  // Squares or products out of fp32's range, or so small that they lost bits.
  if (!finite(top) || top < 1e-30f || (norm && (!finite(sum) || fmaf(sum, inv_k, a.eps) < 1e-30f))) {
    float most = 0.f, none = 0.f;
#pragma unroll
    for (int c = 0; c < kChunks; ++c)
#pragma unroll
      for (int e = 0; e < 8; ++e) most = max_nan(most, fabsf(h[c][e]));
    rt.reduce(none, most);
    if (finite(most) && most > 0.f) {
      // h <- f h, f the power of two that brings the largest into [1, 2), or as near as a factor of 2^100 comes
      const int up = min(100, 127 - max(1, (int)(__float_as_uint(most) >> 23)));
      const float f = up >= -126 ? __uint_as_float((uint32_t)(127 + up) << 23) : __uint_as_float(0x00400000u);   // 2^-127 is denormal
#pragma unroll
      for (int c = 0; c < kChunks; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) h[c][e] *= f;
      measure();
      // w h / sqrt(mean h^2 + eps) = w (f h) / sqrt(mean (f h)^2 + f^2 eps); where f^2 eps passes fp32, the mean is nothing beside it
      const float scaled_eps = a.eps * f * f;
      factor = !norm ? 1.f / f : finite(scaled_eps) ? rsqrtf(fmaf(sum, inv_k, scaled_eps)) : rsqrtf(a.eps) / f;
      divide = true;
    } else if (most == 0.f) {
      factor = 0.f;                                  // a row of zeros stays one, with eps = 0 too
    }
  }
  const bool fine = finite(top);
  const float inv = fine && top > 0.f ? 127.f / top : 0.f;
  if (a.x_q && i == 0) a.scale[t] = fine ? top * factor * (1.f / 127.f) : __uint_as_float(0x7FC00000u);
#pragma unroll
  for (int c = 0; c < kChunks; ++c) {
    const int at = i + c * row_threads;
    if (at >= chunks) continue;
    float w[8];
    weights(at, w);
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] *= h[c][e];
    if (a.y) {
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = w[e] * factor;
      store_eight(reinterpret_cast<T*>(a.y) + t * a.ld_y + at * 8, v);
    }
    if (a.x_q) {
      uint32_t q[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {                  // |w / top| 127 <= 127 (1 + 2^-22): rounds into -127..127
        const float v = divide ? (top > 0.f ? w[e] / top * 127.f : 0.f) : w[e] * inv;
        q[e] = fine ? (uint32_t)__float2int_rn(v) : 0u;
      }
      *reinterpret_cast<uint2*>(a.x_q + t * a.ld_q + at * 8) =
          make_uint2((q[0] & 255u) | (q[1] & 255u) << 8 | (q[2] & 255u) << 16 | q[3] << 24,
                     (q[4] & 255u) | (q[5] & 255u) << 8 | (q[6] & 255u) << 16 | q[7] << 24);
    }
  }
}

template <typename T, int kChunks>
cudaError_t launch_chunks(const NormQuantArgs& a, int row_threads, cudaStream_t s) {
  const int per_block = row_threads >= 128 ? 1 : 128 / row_threads;
  const int64_t blocks = (a.T + per_block - 1) / per_block;
  const auto kern = a.rows ? rms_norm_quant_kernel<T, kChunks, true> : rms_norm_quant_kernel<T, kChunks, false>;
  return launch_pdl(kern, (unsigned)blocks, (unsigned)(row_threads * per_block), 0, s, a, row_threads);
}

template <typename T>
cudaError_t launch_type(const NormQuantArgs& a, cudaStream_t s) {
  const int chunks = (int)(a.K / 8);
  auto threads = [&](int per) { return ((chunks + per - 1) / per + 31) / 32 * 32; };
  if (threads(1) <= 256 || (a.T <= 148 && threads(1) <= 1024)) return launch_chunks<T, 1>(a, threads(1), s);
  if (threads(2) <= 1024) return launch_chunks<T, 2>(a, threads(2), s);
  return launch_chunks<T, 4>(a, threads(4), s);
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
