// Norm of each query and key head with the position rotation, one pass over q and k:
//   x^ = w . x / sqrt(mean x^2 + eps),  (x^_a, x^_b) -> (x^_a cos t - x^_b sin t, x^_b cos t + x^_a sin t).
// Bound by memory: every value is read once and written once.  A head is owned by 8, 16 or 32 lanes, 8
// values per lane (one 16-byte access for 16-bit types); the mean is a shuffle sum over those lanes, a
// rotation partner is either in the lane (interleaved pairs) or rot_dim / 16 lanes away (one shuffle per value).
// A CTA works on one token, so the angles of the token are formed once for all of its heads: position .
// inv_freq / 2 pi in fp64, of which only the fraction of a turn is kept, then sincospif in fp32.  The fp64
// product costs a position of 10^6 nothing; in fp32 its angle would be off by 0.06.  Loads of x are issued
// before the angles are formed.
#include "common.cuh"

namespace bl {

namespace {

constexpr int kNrThreads = 256;
constexpr double kInv2Pi = 0.15915494309189533577;

template <typename T> struct Raw8 { uint4 r; };
template <> struct Raw8<float> { float4 a, b; };

// Plain (coherent) loads: the outputs may be the inputs.
template <typename T> __device__ __forceinline__ Raw8<T> raw_load(const T* p) {
  return Raw8<T>{*reinterpret_cast<const uint4*>(p)};
}
template <> __device__ __forceinline__ Raw8<float> raw_load<float>(const float* p) {
  return Raw8<float>{*reinterpret_cast<const float4*>(p), *reinterpret_cast<const float4*>(p + 4)};
}
__device__ __forceinline__ void raw_floats(const Raw8<float>& x, float (&v)[8]) {
  v[0] = x.a.x; v[1] = x.a.y; v[2] = x.a.z; v[3] = x.a.w; v[4] = x.b.x; v[5] = x.b.y; v[6] = x.b.z; v[7] = x.b.w;
}
__device__ __forceinline__ void raw_floats(const Raw8<__half>& x, float (&v)[8]) {
  const __half2* h = reinterpret_cast<const __half2*>(&x.r);
#pragma unroll
  for (int i = 0; i < 4; ++i) { const float2 f = __half22float2(h[i]); v[2 * i] = f.x; v[2 * i + 1] = f.y; }
}
__device__ __forceinline__ void raw_floats(const Raw8<__nv_bfloat16>& x, float (&v)[8]) {
  const uint32_t* w = reinterpret_cast<const uint32_t*>(&x.r);
#pragma unroll
  for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
  *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void store8(__half* p, const float (&v)[8]) {
  uint4 r;
  __half2* h = reinterpret_cast<__half2*>(&r);
#pragma unroll
  for (int i = 0; i < 4; ++i) h[i] = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
  *reinterpret_cast<uint4*>(p) = r;
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&v)[8]) {
  uint4 r;
  __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&r);
#pragma unroll
  for (int i = 0; i < 4; ++i) h[i] = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
  *reinterpret_cast<uint4*>(p) = r;
}

// kLanes lanes per head (head_dim <= 8 kLanes); a thread takes up to kUnits heads, kNrThreads / kLanes apart.
template <typename T, int kLanes, int kUnits>
__global__ void __launch_bounds__(kNrThreads) qk_norm_rope_kernel(NormRopeArgs a) {
  constexpr int kPerPass = kNrThreads / kLanes;
  __shared__ float2 turn[128];                       // (cos, sin) of the token's pairs
  const int64_t t = blockIdx.x;
  const int sub = threadIdx.x % kLanes, first = blockIdx.y * kUnits * kPerPass + threadIdx.x / kLanes;
  const int d = sub * 8, half = a.rot_dim / 2, heads = a.heads + a.kv_heads;
  const bool on = d < a.head_dim;
  const int pos = a.positions[t];
  if (pos < 0) return;                               // padding: rows stay as they are

  Raw8<T> x[kUnits];
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    const int h = first + u * kPerPass;
    x[u] = Raw8<T>{};
    if (on && h < heads) {
      const T* row = h < a.heads ? reinterpret_cast<const T*>(a.q) + t * a.ld_q + (int64_t)h * a.head_dim
                                 : reinterpret_cast<const T*>(a.k) + t * a.ld_k + (int64_t)(h - a.heads) * a.head_dim;
      x[u] = raw_load(row + d);
    }
  }
  if (threadIdx.x < half) {
    const double turns = (double)pos * (double)a.inv_freq[threadIdx.x] * kInv2Pi;
    float s, c;
    sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
    turn[threadIdx.x] = make_float2(c, s);
  }
  __syncthreads();

  const bool turns_here = d < a.rot_dim;             // rot_dim and d are multiples of 8: a lane turns all of its values or none
  const bool low = d < half;                         // lane holds first members of its pairs (pairs half apart)
  const int lane = threadIdx.x & 31;
  const int partner = (lane - sub) + (!turns_here ? sub : low ? sub + half / 8 : sub - half / 8);
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    const int h = first + u * kPerPass;
    if (__all_sync(0xFFFFFFFFu, h >= heads)) break;
    const bool is_q = h < a.heads;
    float v[8];
    raw_floats(x[u], v);
    if (a.eps >= 0.f) {
      float ss = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) ss = fmaf(v[i], v[i], ss);
#pragma unroll
      for (int o = kLanes / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xFFFFFFFFu, ss, o);
      const float r = 1.0f / sqrtf(ss / (float)a.head_dim + a.eps);
      const T* w = reinterpret_cast<const T*>(is_q ? a.wq : a.wk);
      if (w && on) {
        float g[8];
        Elem<T>::load8(w + d, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = v[i] * r * g[i];
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= r;
      }
    }
    if (a.interleaved) {
      if (turns_here) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 cs = turn[d / 2 + i];
          const float p = v[2 * i], q = v[2 * i + 1];
          v[2 * i] = p * cs.x - q * cs.y;
          v[2 * i + 1] = q * cs.x + p * cs.y;
        }
      }
    } else if (half > 0) {
      const int base = low ? d : d - half;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float other = __shfl_sync(0xFFFFFFFFu, v[i], partner);
        if (turns_here) {
          const float2 cs = turn[base + i];
          v[i] = low ? v[i] * cs.x - other * cs.y : v[i] * cs.x + other * cs.y;
        }
      }
    }
    if (on && h < heads) {
      T* row = is_q ? reinterpret_cast<T*>(a.q_out) + t * a.ld_qo + (int64_t)h * a.head_dim
                    : reinterpret_cast<T*>(a.k_out) + t * a.ld_ko + (int64_t)(h - a.heads) * a.head_dim;
      store8(row + d, v);
    }
  }
}

template <typename T, int kLanes>
cudaError_t launch_lanes(const NormRopeArgs& a, cudaStream_t s) {
  constexpr int kPerPass = kNrThreads / kLanes;
  const int heads = a.heads + a.kv_heads;
  const int passes = (heads + kPerPass - 1) / kPerPass;
  // few tokens: one pass per CTA, so that the heads of a token spread over the SMs; many: up to four, so
  // that the angles of a token are formed for up to four passes of heads at once
  if (a.T * passes <= 4 * 148) {
    qk_norm_rope_kernel<T, kLanes, 1><<<dim3((unsigned)a.T, (unsigned)passes), kNrThreads, 0, s>>>(a);
  } else {
    qk_norm_rope_kernel<T, kLanes, 4><<<dim3((unsigned)a.T, (unsigned)((passes + 3) / 4)), kNrThreads, 0, s>>>(a);
  }
  return cudaGetLastError();
}

template <typename T>
cudaError_t launch_type(const NormRopeArgs& a, cudaStream_t s) {
  if (a.head_dim <= 64) return launch_lanes<T, 8>(a, s);
  if (a.head_dim <= 128) return launch_lanes<T, 16>(a, s);
  return launch_lanes<T, 32>(a, s);
}

}  // namespace

cudaError_t launch_qk_norm_rope(const NormRopeArgs& a, cudaStream_t s) {
  switch (a.dt) {
    case BL_F32: return launch_type<float>(a, s);
    case BL_F16: return launch_type<__half>(a, s);
    default: return launch_type<__nv_bfloat16>(a, s);
  }
}

}  // namespace bl
