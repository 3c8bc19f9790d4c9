// Attention of prompts with a sliding window and sinks (bitlinear_attention_window).
// One warp per (query row, head): a pass over the visible keys with the running maximum and sum of the
// softmax, each lane holding kDim / 32 values of the query and of the output.
#include "common.cuh"

namespace bl {

namespace {

// Rows of one sequence in q / o and in k / v.
struct SeqRows { int q0, nq, k0, nk; };
__device__ __forceinline__ SeqRows seq_rows(const WindowArgs& a, int b) {
  SeqRows r;
  if (a.cu_q) {
    r.q0 = min(max(a.cu_q[b], 0), (int)a.rows_q);
    r.nq = min(min(max(a.cu_q[b + 1], r.q0), (int)a.rows_q) - r.q0, (int)a.seq_q);
    r.k0 = min(max(a.cu_k[b], 0), (int)a.rows_k);
    r.nk = min(min(max(a.cu_k[b + 1], r.k0), (int)a.rows_k) - r.k0, (int)a.seq_k);
  } else {
    r.q0 = b * (int)a.seq_q; r.nq = (int)a.seq_q;
    r.k0 = b * (int)a.seq_k; r.nk = (int)a.seq_k;
  }
  return r;
}

// Query row i (of r.nq) of head h, by one warp.
template <typename T, int kDim>
__device__ void window_row(const WindowArgs& a, const SeqRows& r, int i, int h) {
  constexpr int kVals = kDim / 32;
  const int lane = threadIdx.x & 31, hk = h / (a.heads / a.kv_heads), pos = r.nk - r.nq + i;
  const T* q = reinterpret_cast<const T*>(a.q) + (int64_t)(r.q0 + i) * a.ld_q + (int64_t)h * kDim + lane * kVals;
  const T* k = reinterpret_cast<const T*>(a.k) + (int64_t)r.k0 * a.ld_k + (int64_t)hk * kDim + lane * kVals;
  const T* v = reinterpret_cast<const T*>(a.v) + (int64_t)r.k0 * a.ld_v + (int64_t)hk * kDim + lane * kVals;
  float qv[kVals], acc[kVals];
#pragma unroll
  for (int e = 0; e < kVals; ++e) { qv[e] = in_cast(q[e]); acc[e] = 0.f; }
  float m = -INFINITY, l = 0.f;
  for (int j = 0; j <= pos; ++j) {
    if (a.window > 0 && pos - j >= a.window && j >= a.sinks) continue;
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < kVals; ++e) s = fmaf(qv[e], in_cast(k[(int64_t)j * a.ld_k + e]), s);
    s = warp_sum(s) * a.scale;
    const float top = fmaxf(m, s), c = m == -INFINITY ? 0.f : expf(m - top), p = expf(s - top);
    m = top;
    l = l * c + p;
#pragma unroll
    for (int e = 0; e < kVals; ++e) acc[e] = acc[e] * c + p * in_cast(v[(int64_t)j * a.ld_v + e]);
  }
  T* o = reinterpret_cast<T*>(a.o) + (int64_t)(r.q0 + i) * a.ld_o + (int64_t)h * kDim + lane * kVals;
#pragma unroll
  for (int e = 0; e < kVals; ++e) o[e] = out_cast<T>(l == 0.f ? 0.f : acc[e] / l);
}

// One CTA per (128 query rows, head, sequence), four warps.
template <typename T, int kDim>
__global__ void __launch_bounds__(128) attention_window_kernel(WindowArgs a) {
  const int tiles = (int)((a.seq_q + 127) / 128);
  const int tile = blockIdx.x % tiles, h = blockIdx.x / tiles % a.heads, b = blockIdx.x / tiles / a.heads;
  const SeqRows r = seq_rows(a, b);
  const int last = min(tile * 128 + 128, r.nq);
  for (int i = tile * 128 + (threadIdx.x >> 5); i < last; i += 4) window_row<T, kDim>(a, r, i, h);
}

template <typename T>
cudaError_t launch_type(const WindowArgs& a, cudaStream_t s) {
  const unsigned grid = (unsigned)((a.seq_q + 127) / 128 * a.heads * a.batch);
  if (a.head_dim == 64) attention_window_kernel<T, 64><<<grid, 128, 0, s>>>(a);
  else attention_window_kernel<T, 128><<<grid, 128, 0, s>>>(a);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_attention_window(const WindowArgs& a, cudaStream_t s) {
  return a.dt == BL_F16 ? launch_type<__half>(a, s) : launch_type<__nv_bfloat16>(a, s);
}

}  // namespace bl
