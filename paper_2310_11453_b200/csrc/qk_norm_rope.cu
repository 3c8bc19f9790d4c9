// Norm of each query and key head with the position rotation, one pass over q and k:
//   x^ = w . x / sqrt(mean x^2 + eps),  (x^_a, x^_b) -> (x^_a cos t - x^_b sin t, x^_b cos t + x^_a sin t).
// Bound by memory: every value is read once and written once.  A head is owned by 8, 16 or 32 lanes.  A lane holds
// two runs of four values that contain both members of its four pairs (i.. and rot_dim / 2 + i.., or neighbours when
// interleaved), so the rotation needs no exchange, and the same places of every head it works on, so that cos, sin and
// the weights of those places stay in registers.  Only the mean takes shuffles.
// A warp works on one token and a run of its heads, kAhead loads in flight, with no barrier.  The angles are formed
// once per warp: position . inv_freq / 2 pi in fp64, of which only the fraction of a turn is kept, then sincospif in
// fp32 (in fp32 alone the angle of position 10^6 would be off by 0.06).
#include "common.cuh"

namespace bl {

namespace {

constexpr int kNrWarps = 4;
constexpr int kAhead = 4;                          // heads per lane group loaded ahead
constexpr double kInv2Pi = 0.15915494309189533577;

template <typename T> struct Quad { uint2 r; };    // four values as stored
template <> struct Quad<float> { float4 r; };
template <typename T> __device__ __forceinline__ Quad<T> load_quad(const T* p) {       // coherent: outputs may be the inputs
  Quad<T> q;
  q.r = *reinterpret_cast<const decltype(q.r)*>(p);
  return q;
}
__device__ __forceinline__ void floats(const Quad<float>& q, float* v) { v[0] = q.r.x; v[1] = q.r.y; v[2] = q.r.z; v[3] = q.r.w; }
__device__ __forceinline__ void floats(const Quad<__half>& q, float* v) {
  const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&q.r.x)), b = __half22float2(*reinterpret_cast<const __half2*>(&q.r.y));
  v[0] = a.x; v[1] = a.y; v[2] = b.x; v[3] = b.y;
}
__device__ __forceinline__ void floats(const Quad<__nv_bfloat16>& q, float* v) {
  v[0] = __uint_as_float(q.r.x << 16); v[1] = __uint_as_float(q.r.x & 0xFFFF0000u);
  v[2] = __uint_as_float(q.r.y << 16); v[3] = __uint_as_float(q.r.y & 0xFFFF0000u);
}
__device__ __forceinline__ void store_quad(float* p, const float* v) { *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]); }
__device__ __forceinline__ void store_quad(__half* p, const float* v) {
  uint2 r;
  *reinterpret_cast<__half2*>(&r.x) = __floats2half2_rn(v[0], v[1]);
  *reinterpret_cast<__half2*>(&r.y) = __floats2half2_rn(v[2], v[3]);
  *reinterpret_cast<uint2*>(p) = r;
}
__device__ __forceinline__ void store_quad(__nv_bfloat16* p, const float* v) {
  uint2 r;
  *reinterpret_cast<__nv_bfloat162*>(&r.x) = __floats2bfloat162_rn(v[0], v[1]);
  *reinterpret_cast<__nv_bfloat162*>(&r.y) = __floats2bfloat162_rn(v[2], v[3]);
  *reinterpret_cast<uint2*>(p) = r;
}

// kLanes lanes per head (head_dim <= 8 kLanes).  Warp (token, part) takes heads part * per .. of the token's query and
// key heads in one row of numbers.
template <typename T, int kLanes>
__global__ void __launch_bounds__(kNrWarps * 32) qk_norm_rope_kernel(NormRopeArgs a, int parts, int per) {
  constexpr int kGroups = 32 / kLanes;
  const int lane = threadIdx.x & 31, sub = lane % kLanes, group = lane / kLanes;
  const int64_t job = (int64_t)blockIdx.x * kNrWarps + (threadIdx.x >> 5);
  const int64_t t = job / parts;
  if (t >= a.T) return;
  const int heads = a.heads + a.kv_heads, h0 = (int)(job - t * parts) * per, h1 = min(h0 + per, heads);
  const int pos = a.positions[t];
  if (pos < 0 || h0 >= h1) return;                 // padding: rows stay as they are
  const int half = a.rot_dim / 2;
  const bool on = sub * 8 < a.head_dim, turns = sub * 8 < a.rot_dim;
  // where this lane's two runs of four lie in a head, and its first pair
  const int d0 = a.interleaved || !turns ? sub * 8 : sub * 4;
  const int d1 = a.interleaved || !turns ? sub * 8 + 4 : half + sub * 4;

  const T* q = reinterpret_cast<const T*>(a.q) + t * a.ld_q;
  const T* k = reinterpret_cast<const T*>(a.k) + t * a.ld_k;
  Quad<T> x[kAhead][2];
  auto fetch = [&](int h, Quad<T> (&r)[2]) {
    r[0] = Quad<T>{}; r[1] = Quad<T>{};
    if (on && h < h1) {
      const T* row = h < a.heads ? q + (int64_t)h * a.head_dim : k + (int64_t)(h - a.heads) * a.head_dim;
      r[0] = load_quad(row + d0);
      r[1] = load_quad(row + d1);
    }
  };
#pragma unroll
  for (int i = 0; i < kAhead; ++i) fetch(h0 + i * kGroups + group, x[i]);

  // cos and sin of the token's pairs: lane i forms those of pairs i, i + 32, .., then hands them out
  float c[4], s[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) { c[i] = 1.f; s[i] = 0.f; }
  for (int base = 0; base < half; base += 32) {
    float cl = 1.f, sl = 0.f;
    if (base + lane < half) {
      const double turn = (double)pos * (double)a.inv_freq[base + lane] * kInv2Pi;
      sincospif(2.f * (float)(turn - rint(turn)), &sl, &cl);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int pair = sub * 4 + i - base;
      const float ci = __shfl_sync(0xFFFFFFFFu, cl, pair & 31), si = __shfl_sync(0xFFFFFFFFu, sl, pair & 31);
      if (turns && pair >= 0 && pair < 32) { c[i] = ci; s[i] = si; }
    }
  }
  const bool norm = a.eps >= 0.f;
  Quad<T> wq[2] = {}, wk[2] = {};
  if (on && norm) {
    if (a.wq) { wq[0] = load_quad(reinterpret_cast<const T*>(a.wq) + d0); wq[1] = load_quad(reinterpret_cast<const T*>(a.wq) + d1); }
    if (a.wk) { wk[0] = load_quad(reinterpret_cast<const T*>(a.wk) + d0); wk[1] = load_quad(reinterpret_cast<const T*>(a.wk) + d1); }
  }
  const float inv_dim = 1.f / (float)a.head_dim;

  for (int base = h0; base < h1; base += kAhead * kGroups) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int h = base + i * kGroups + group;
      const bool is_q = h < a.heads;
      float v[8];
      floats(x[i][0], v);
      floats(x[i][1], v + 4);
      fetch(h + kAhead * kGroups, x[i]);
      if (norm) {
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = fmaf(v[e], v[e], ss);
#pragma unroll
        for (int o = kLanes / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xFFFFFFFFu, ss, o);
        const float r = 1.0f / sqrtf(fmaf(ss, inv_dim, a.eps));
        if (is_q ? a.wq != nullptr : a.wk != nullptr) {
          float g[8];
          floats(is_q ? wq[0] : wk[0], g);
          floats(is_q ? wq[1] : wk[1], g + 4);
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = v[e] * r * g[e];
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] *= r;
        }
      }
      float y[8];
      if (a.interleaved) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          y[2 * e] = v[2 * e] * c[e] - v[2 * e + 1] * s[e];
          y[2 * e + 1] = v[2 * e + 1] * c[e] + v[2 * e] * s[e];
        }
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          y[e] = v[e] * c[e] - v[4 + e] * s[e];
          y[4 + e] = v[4 + e] * c[e] + v[e] * s[e];
        }
      }
      if (on && h < h1) {
        T* row = is_q ? reinterpret_cast<T*>(a.q_out) + t * a.ld_qo + (int64_t)h * a.head_dim
                      : reinterpret_cast<T*>(a.k_out) + t * a.ld_ko + (int64_t)(h - a.heads) * a.head_dim;
        store_quad(row + d0, y);
        store_quad(row + d1, y + 4);
      }
    }
  }
}

template <typename T, int kLanes>
cudaError_t launch_lanes(const NormRopeArgs& a, cudaStream_t s) {
  constexpr int kStep = kAhead * (32 / kLanes);      // heads a warp has in flight
  const int heads = a.heads + a.kv_heads;
  // Few tokens: as little as one load per lane and warp, so that the heads spread over the SMs.  Many: runs of about 20
  // heads, over which a warp's angles and weights are used again.
  const int most = (heads + kStep - 1) / kStep * kStep;
  int per = (heads + (heads + 23) / 24 - 1) / ((heads + 23) / 24);
  if (a.T * ((heads + per - 1) / per) < 148 * 16) per = 32 / kLanes;
  per = per < most ? per : most;
  const int parts = (heads + per - 1) / per;
  const int64_t blocks = (a.T * parts + kNrWarps - 1) / kNrWarps;
  if (blocks > 0x7FFFFFFF) return cudaErrorInvalidValue;
  qk_norm_rope_kernel<T, kLanes><<<(unsigned)blocks, kNrWarps * 32, 0, s>>>(a, parts, per);
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
