// Attention of the last n_q tokens of each sequence over the 4-bit paged cache.
// One warp per (sequence, query, head): a pass over the visible tokens with the running maximum and sum of the
// softmax, each lane holding kDim / 32 values of the query and of the output.
#include "kv4.cuh"

namespace bl {

namespace {

using namespace kv4;

template <typename T, int kDim>
__global__ void __launch_bounds__(128) attention_kv4_kernel(Kv4AttnArgs a) {
  constexpr int kVals = kDim / 32;
  const int lane = threadIdx.x & 31;
  const int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
  if (w >= (int64_t)a.batch * a.n_q * a.heads) return;
  const int h = (int)(w % a.heads), hk = h / (a.heads / a.cache.kv_heads);
  const int64_t row = w / a.heads;
  const int b = (int)(row / a.n_q), i = (int)(row % a.n_q);
  const int ps = a.cache.page_size;
  const int len = (int)min((int64_t)max(a.lens[b], 0), a.max_pages * ps);
  const int pos = len - a.n_q + i;
  const T* q = reinterpret_cast<const T*>(a.q) + row * a.ld_q + (int64_t)h * kDim + lane * kVals;
  float qv[kVals], acc[kVals];
#pragma unroll
  for (int e = 0; e < kVals; ++e) { qv[e] = in_cast(q[e]); acc[e] = 0.f; }
  float m = -INFINITY, l = 0.f;
  for (int j = 0; j <= pos; ++j) {
    if (a.window > 0 && pos - j >= a.window && j >= a.sinks) continue;
    const int page = a.table[(int64_t)b * a.max_pages + j / ps];
    if (page < 0 || page >= a.cache.num_pages) continue;
    const char* block = reinterpret_cast<const char*>(a.cache.pages) + ((int64_t)page * a.cache.kv_heads + hk) * Block<kDim>::bytes(ps);
    const int t = j % ps;
    const float2 ks = scale_floats<T>(*reinterpret_cast<const uint32_t*>(block + Block<kDim>::k_scale(ps) + 4 * t));
    const float2 vs = scale_floats<T>(*reinterpret_cast<const uint32_t*>(block + Block<kDim>::v_scale(ps) + 4 * t));
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < kVals; ++e) {
      const int d = lane * kVals + e;
      const int code = ((uint8_t)block[t * (kDim / 2) + d / 2] >> (4 * (d & 1))) & 15;
      s = fmaf(qv[e], fmaf((float)code, ks.x, ks.y), s);
    }
    s = warp_sum(s) * a.scale;
    const float top = fmaxf(m, s), c = m == -INFINITY ? 0.f : expf(m - top), p = expf(s - top);
    m = top;
    l = l * c + p;
#pragma unroll
    for (int e = 0; e < kVals; ++e) {
      const int d = lane * kVals + e;
      const uint8_t byte = (uint8_t)block[Block<kDim>::v_codes(ps) + Block<kDim>::v_at(t, d & ~3) + ((d & 3) >> 1)];
      acc[e] = acc[e] * c + p * fmaf((float)((byte >> (4 * (d & 1))) & 15), vs.x, vs.y);
    }
  }
  T* o = reinterpret_cast<T*>(a.o) + row * a.ld_o + (int64_t)h * kDim + lane * kVals;
#pragma unroll
  for (int e = 0; e < kVals; ++e) o[e] = out_cast<T>(l == 0.f ? 0.f : acc[e] / l);
}

template <typename T>
cudaError_t launch_type(const Kv4AttnArgs& a, cudaStream_t s) {
  const unsigned grid = (unsigned)(((int64_t)a.batch * a.n_q * a.heads + 3) / 4);
  if (a.cache.head_dim == 64) attention_kv4_kernel<T, 64><<<grid, 128, 0, s>>>(a);
  else attention_kv4_kernel<T, 128><<<grid, 128, 0, s>>>(a);
  return cudaGetLastError();
}

}  // namespace

size_t attention_kv4_ws_bytes(int, int, int, int, int) { return 256; }

cudaError_t launch_attention_kv4(const Kv4AttnArgs& a, cudaStream_t s) {
  return a.cache.dtype == BL_F16 ? launch_type<__half>(a, s) : launch_type<__nv_bfloat16>(a, s);
}

}  // namespace bl
