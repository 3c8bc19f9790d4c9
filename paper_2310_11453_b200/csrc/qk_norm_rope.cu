// Norm of each query and key head with the position rotation, one pass over q and k:
//   x^ = w . x / sqrt(mean x^2 + eps),  (x^_a, x^_b) -> (x^_a cos t - x^_b sin t, x^_b cos t + x^_a sin t).
// Bound by memory: every value is read once and written once.  A lane owns 16 values of a head: two runs of eight that
// contain both members of its eight pairs (8 i.. and rot_dim / 2 + 8 i.., or 16 neighbours when interleaved), so the
// rotation needs no exchange, and the same places of every head it works on, so that cos, sin and the weights of those
// places stay in registers.  Only the mean takes shuffles, over the 4, 8 or 16 lanes of a head.
// A warp works on one token and a run of its heads, kAhead loads in flight, with no barrier.  The angles are formed
// once per warp: position . inv_freq / 2 pi in fp64, of which only the fraction of a turn is kept, then sincospif in
// fp32 (in fp32 alone the angle of position 10^6 would be off by 0.06).
#include "common.cuh"

namespace bl {

namespace {

constexpr int kNrWarps = 4;
constexpr int kAhead = 2;                          // heads per lane group loaded ahead
constexpr double kInv2Pi = 0.15915494309189533577;

template <typename T> struct Run { uint4 r; };     // eight values as stored
template <> struct Run<float> { float4 a, b; };
template <typename T> __device__ __forceinline__ Run<T> load_run(const T* p) {         // coherent: outputs may be the inputs
  return Run<T>{*reinterpret_cast<const uint4*>(p)};
}
template <> __device__ __forceinline__ Run<float> load_run<float>(const float* p) {
  return Run<float>{*reinterpret_cast<const float4*>(p), *reinterpret_cast<const float4*>(p + 4)};
}
__device__ __forceinline__ void floats(const Run<float>& q, float* v) {
  v[0] = q.a.x; v[1] = q.a.y; v[2] = q.a.z; v[3] = q.a.w; v[4] = q.b.x; v[5] = q.b.y; v[6] = q.b.z; v[7] = q.b.w;
}
__device__ __forceinline__ void floats(const Run<__half>& q, float* v) {
  const __half2* h = reinterpret_cast<const __half2*>(&q.r);
#pragma unroll
  for (int i = 0; i < 4; ++i) { const float2 f = __half22float2(h[i]); v[2 * i] = f.x; v[2 * i + 1] = f.y; }
}
__device__ __forceinline__ void floats(const Run<__nv_bfloat16>& q, float* v) {
  const uint32_t w[4] = {q.r.x, q.r.y, q.r.z, q.r.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
}
__device__ __forceinline__ void store_run(float* p, const float* v) {
  *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void store_run(__half* p, const float* v) {
  uint4 r;
  __half2* h = reinterpret_cast<__half2*>(&r);
#pragma unroll
  for (int i = 0; i < 4; ++i) h[i] = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
  *reinterpret_cast<uint4*>(p) = r;
}
__device__ __forceinline__ void store_run(__nv_bfloat16* p, const float* v) {
  uint4 r;
  __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&r);
#pragma unroll
  for (int i = 0; i < 4; ++i) h[i] = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
  *reinterpret_cast<uint4*>(p) = r;
}

// One of q and k as a warp's job sees it: the token's rows, and the heads to take.
template <typename T> struct Heads { const T* in; T* out; const T* w; int from, to; };

template <typename T, int kLanes, bool kInter, bool kWhole>
__device__ __forceinline__ void turn_heads(const Heads<T>& x, const NormRopeArgs& a, const float (&c)[8], const float (&s)[8], bool on,
                                           bool turns, int d0, int d1) {
  constexpr int kGroups = 32 / kLanes;
  const int group = (threadIdx.x & 31) / kLanes;
  const bool norm = a.eps >= 0.f, weigh = norm && x.w != nullptr;
  Run<T> r[kAhead][2];
  auto fetch = [&](int h, Run<T> (&y)[2]) {
    y[0] = Run<T>{}; y[1] = Run<T>{};
    if (on && h < x.to) {
      y[0] = load_run(x.in + (int64_t)h * a.head_dim + d0);
      y[1] = load_run(x.in + (int64_t)h * a.head_dim + d1);
    }
  };
#pragma unroll
  for (int i = 0; i < kAhead; ++i) fetch(x.from + i * kGroups + group, r[i]);
  float g[16];
#pragma unroll
  for (int e = 0; e < 16; ++e) g[e] = 1.f;
  if (on && weigh) { floats(load_run(x.w + d0), g); floats(load_run(x.w + d1), g + 8); }
  const float inv_dim = 1.f / (float)a.head_dim;
  for (int base = x.from; base < x.to; base += kAhead * kGroups) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int h = base + i * kGroups + group;
      float v[16];
      floats(r[i][0], v);
      floats(r[i][1], v + 8);
      fetch(h + kAhead * kGroups, r[i]);
      if (norm) {
        float s0 = 0.f, s1 = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) { s0 = fmaf(v[e], v[e], s0); s1 = fmaf(v[8 + e], v[8 + e], s1); }
        float ss = s0 + s1;
#pragma unroll
        for (int o = kLanes / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xFFFFFFFFu, ss, o);
        const float f = rsqrtf(fmaf(ss, inv_dim, a.eps));
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] = v[e] * f * g[e];
      }
      if (kWhole || turns) {                         // not by a turn of 0: infinity x 0 would make NaN of the other member
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int p = kInter ? 2 * e : e, q = kInter ? 2 * e + 1 : 8 + e;
          const float vp = v[p], vq = v[q];
          v[p] = vp * c[e] - vq * s[e];
          v[q] = vq * c[e] + vp * s[e];
        }
      }
      if (on && h < x.to) {
        store_run(x.out + (int64_t)h * a.head_dim + d0, v);
        store_run(x.out + (int64_t)h * a.head_dim + d1, v + 8);
      }
    }
  }
}

// kLanes lanes per head (head_dim <= 16 kLanes).  kWhole: the whole head turns, so no lane has to ask (8191 tokens, 32 + 8 heads of
// 128: 32.1 us against 32.7; 16 + 16 heads of 64: 13.9 against 14.8).  Warp (token, part) takes heads part * per .. of the token's query and
// key heads in one row of numbers.
template <typename T, int kLanes, bool kInter, bool kWhole>
__global__ void __launch_bounds__(kNrWarps * 32, sizeof(T) == 2 ? 5 : 4) qk_norm_rope_kernel(NormRopeArgs a, int parts, int per) {
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31, sub = lane % kLanes;
  const int64_t job = (int64_t)blockIdx.x * kNrWarps + (threadIdx.x >> 5);
  const int64_t t = parts == 1 ? job : job / parts;
  if (t >= a.T) return;
  const int h0 = (int)(job - t * parts) * per, h1 = min(h0 + per, a.heads + a.kv_heads);
  pdl_wait();
  const int pos = a.positions[t];
  if (pos < 0) return;                             // padding: rows stay as they are
  const int half = a.rot_dim / 2;
  const bool on = sub * 16 < a.head_dim, turns = sub * 16 < a.rot_dim;
  // where this lane's two runs of eight lie in a head
  const int d0 = kInter || !turns ? sub * 16 : sub * 8, d1 = kInter || !turns ? sub * 16 + 8 : half + sub * 8;
  // cos and sin of the token's pairs: lane i forms those of pairs i, i + 32, .., then hands them out
  float c[8], s[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) { c[i] = 1.f; s[i] = 0.f; }
  for (int base = 0; base < half; base += 32) {
    float cl = 1.f, sl = 0.f;
    if (base + lane < half) {
      const double turn = (double)pos * (double)a.inv_freq[base + lane] * kInv2Pi;
      sincospif(2.f * (float)(turn - rint(turn)), &sl, &cl);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int pair = sub * 8 + i - base;
      const float ci = __shfl_sync(0xFFFFFFFFu, cl, pair & 31), si = __shfl_sync(0xFFFFFFFFu, sl, pair & 31);
      if (turns && pair >= 0 && pair < 32) { c[i] = ci; s[i] = si; }
    }
  }
  const Heads<T> q{reinterpret_cast<const T*>(a.q) + t * a.ld_q, reinterpret_cast<T*>(a.q_out) + t * a.ld_qo,
                   reinterpret_cast<const T*>(a.wq), h0, min(h1, a.heads)};
  const Heads<T> k{reinterpret_cast<const T*>(a.k) + t * a.ld_k, reinterpret_cast<T*>(a.k_out) + t * a.ld_ko,
                   reinterpret_cast<const T*>(a.wk), max(h0 - a.heads, 0), h1 - a.heads};
#pragma unroll 1
  for (int which = 0; which < 2; ++which) {        // one copy of the loop for both
    const Heads<T> x = which ? k : q;
    if (x.from < x.to) turn_heads<T, kLanes, kInter, kWhole>(x, a, c, s, on, turns, d0, d1);
  }
}

template <typename T, int kLanes>
cudaError_t launch_lanes(const NormRopeArgs& a, cudaStream_t s) {
  const int heads = a.heads + a.kv_heads, each = 32 / kLanes;       // heads a warp works on at a time
  // Many tokens: a warp takes all heads of a token, or runs of up to 48, over which its angles and weights serve.  Few: as
  // little as one load per lane, so that the heads spread over the SMs.
  int per = (heads + (heads + 47) / 48 - 1) / ((heads + 47) / 48);
  if (a.T * ((heads + per - 1) / per) < 148 * 16) per = each;
  const int parts = (heads + per - 1) / per;
  const int64_t blocks = (a.T * parts + kNrWarps - 1) / kNrWarps;
  if (blocks > 0x7FFFFFFF) return cudaErrorInvalidValue;
  const auto whole = a.interleaved ? qk_norm_rope_kernel<T, kLanes, true, true> : qk_norm_rope_kernel<T, kLanes, false, true>;
  const auto part = a.interleaved ? qk_norm_rope_kernel<T, kLanes, true, false> : qk_norm_rope_kernel<T, kLanes, false, false>;
  return launch_pdl(a.rot_dim == a.head_dim ? whole : part, (unsigned)blocks, kNrWarps * 32, 0, s, a, parts, per);
}

template <typename T>
cudaError_t launch_type(const NormRopeArgs& a, cudaStream_t s) {
  if (a.head_dim <= 64) return launch_lanes<T, 4>(a, s);
  if (a.head_dim <= 128) return launch_lanes<T, 8>(a, s);
  return launch_lanes<T, 16>(a, s);
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
