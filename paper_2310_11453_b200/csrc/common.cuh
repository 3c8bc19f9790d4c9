// Shared device helpers and the internal launch interface of the BitLinear CUDA library.
// sm_100a only.  Nothing here is used by the CPU oracle.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "../../include/bitlinear.h"

namespace bl {

// Test hook behind bitlinear_debug_wait_limit (defined in api.cu, read by the launchers when a
// call is made): cap on the polls of the bounded device-side waits (negative: built-in limits),
// and whether the cooperative LN+quant kernel waits for a tag that nobody publishes.
extern std::atomic<long long> g_debug_wait_polls;
extern std::atomic<int> g_debug_meet_skew;

// The start of a workspace is what bitlinear_ws_status reads: a status word, 0 or a bl_status, or kStatusPerWarp plus the number
// of such words that follow it, one per warp of the kernel.  The latter is for a kernel whose warps all may report and which
// nothing runs in front of: each warp clears its own word and sets it, so that no report can be cleared by another warp.
constexpr uint32_t kStatusPerWarp = 0x5A570000u;
constexpr uint32_t kMostStatusWords = 2047;

// Programmatic dependent launch.  A kernel launched through launch_pdl() may be scheduled while
// the kernel before it on the stream is still running: it calls pdl_wait() before its first
// access to global memory (after set-up that touches only its own shared memory), which blocks
// until everything earlier on the stream has completed and is visible.  pdl_launch_dependents()
// lets the kernel after this one be scheduled early in the same way.
#ifdef __CUDACC__
__device__ __forceinline__ void pdl_launch_dependents() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

template <typename... KArgs, typename... Args>
inline cudaError_t launch_pdl_clusters(void (*kernel)(KArgs...), dim3 grid, unsigned cluster, unsigned block, size_t smem, cudaStream_t s,
                                       Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(block);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 0 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...);
}
// How many clusters of such a launch the GPU holds at once.
template <typename... KArgs>
inline cudaError_t max_clusters(void (*kernel)(KArgs...), unsigned cluster, unsigned block, size_t smem, int* n) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(cluster);
  cfg.blockDim = dim3(block);
  cfg.dynamicSmemBytes = smem;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cluster;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaOccupancyMaxActiveClusters(n, kernel, &cfg);
}
template <typename... KArgs, typename... Args>
inline cudaError_t launch_pdl(void (*kernel)(KArgs...), dim3 grid, unsigned block, size_t smem, cudaStream_t s,
                              Args... args) {
  return launch_pdl_clusters(kernel, grid, 0, block, smem, s, args...);
}
#endif

constexpr int kQb = 128;             // Q_b = 2^(b-1), b = 8
constexpr int kCodeMax = kQb - 1;    // Clip bound with the paper's eps taken as one code
constexpr float kInvQb = 1.0f / 128.0f;

// ---- element loads: 8 consecutive elements of a 16-byte aligned row as floats ------------
template <typename T> struct Elem;
template <> struct Elem<float> {
  static __device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
    float4 a = __ldg(reinterpret_cast<const float4*>(p));
    float4 b = __ldg(reinterpret_cast<const float4*>(p) + 1);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  }
  static __device__ __forceinline__ float to_out(float f) { return f; }
};
template <> struct Elem<__half> {
  static __device__ __forceinline__ void load8(const __half* p, float (&v)[8]) {
    uint4 r = __ldg(reinterpret_cast<const uint4*>(p));
    const __half2* h = reinterpret_cast<const __half2*>(&r);
#pragma unroll
    for (int i = 0; i < 4; ++i) { float2 f = __half22float2(h[i]); v[2 * i] = f.x; v[2 * i + 1] = f.y; }
  }
  static __device__ __forceinline__ __half to_out(float f) { return __float2half_rn(f); }
};
template <> struct Elem<__nv_bfloat16> {
  static __device__ __forceinline__ void load8(const __nv_bfloat16* p, float (&v)[8]) {
    uint4 r = __ldg(reinterpret_cast<const uint4*>(p));
    const uint32_t* w = reinterpret_cast<const uint32_t*>(&r);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
  static __device__ __forceinline__ __nv_bfloat16 to_out(float f) { return __float2bfloat16_rn(f); }
};

// ---- order-preserving float <-> uint encoding for atomic min/max ---------------------------
__device__ __forceinline__ uint32_t enc_ordered(float f) {
  uint32_t b = __float_as_uint(f);
  return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ float dec_ordered(uint32_t e) {
  uint32_t b = (e & 0x80000000u) ? (e & 0x7FFFFFFFu) : ~e;
  return __uint_as_float(b);
}

// ---- warp / block reductions (fixed order, deterministic) ---------------------------------
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
  return v;
}
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
  return v;
}
__device__ __forceinline__ float warp_min(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = fminf(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
  return v;
}
__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
  return v;
}
__device__ __forceinline__ int warp_sum(int v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
  return v;
}

// ---- Quant of one normalised value, Eq. 4-6 (round-half-to-even, then clip) ----------------
// scale = Q_b / gamma (0 when gamma == 0); shift = eta (0 for absmax); lo = -127 or 0.
__device__ __forceinline__ int quant_code(float xhat, float shift, float scale, int lo) {
  int c = __float2int_rn((xhat - shift) * scale);
  return max(lo, min(kCodeMax, c));
}

// ---- Eq. 11 rescale of one group's integer sum (shared by every matmul kernel) --------------
// acc * beta_g * gamma / Q_b, plus eta * beta_g * rowsum when the eta shift is undone.
__device__ __forceinline__ float dequant_term(int acc, float beta_g, float gamma, float eta,
                                              int rowsum, bool correct) {
  float v = (float)acc * (beta_g * gamma * kInvQb);
  if (correct) v += eta * beta_g * (float)rowsum;
  return v;
}

__device__ __forceinline__ float in_cast(float v) { return v; }
__device__ __forceinline__ float in_cast(__half v) { return __half2float(v); }
__device__ __forceinline__ float in_cast(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T out_cast(float f);
template <> __device__ __forceinline__ float out_cast<float>(float f) { return f; }
template <> __device__ __forceinline__ __half out_cast<__half>(float f) { return __float2half_rn(f); }
template <> __device__ __forceinline__ __nv_bfloat16 out_cast<__nv_bfloat16>(float f) { return __float2bfloat16_rn(f); }

// ---- internal launchers (defined one per .cu file) -----------------------------------------
struct PackArgs {
  const void* W; bl_dtype wt; int64_t N, K; int G; bl_layout layout; const float* alpha_in;
  uint8_t* W_packed; float* alpha; float* beta; int32_t* rowsum; void* ws;
};
size_t pack_ws_bytes(int G);
cudaError_t launch_binarize_pack(const PackArgs& a, cudaStream_t s);

struct QuantArgs {
  const void* x; bl_dtype xt; int64_t M, K; int G; bl_quant_mode mode; bl_gran gran; float ln_eps;
  int8_t* x_q; float* gamma; float* eta; void* ws;
  uint32_t* status = nullptr;                      // word for a device-side timeout.  nullptr: per-tensor
                                                   // scope uses the first word of ws, per-token scope runs
                                                   // without bounded waits (per-lane copies)
  int keep_status = 0;                             // an earlier kernel of the call already cleared the word
};
size_t quant_ws_bytes(int64_t M, int G);
cudaError_t launch_quant_act(const QuantArgs& a, cudaStream_t s);

// Integer matmul, optionally with the Eq. 11 rescale fused.  When y != nullptr the kernel
// writes y (dtype yt); otherwise it writes acc [G,M,N].
struct GemmArgs {
  const int8_t* x_q; int64_t M, K, N; int G; const uint8_t* W_packed;
  int32_t* acc;                                    // int32 output, or nullptr
  void* y; bl_dtype yt;                            // dequantised output, or nullptr
  const float* beta; const float* gamma; const float* eta; bl_gran gran;
  const int32_t* rowsum; int eta_correction;
  // Epilogue options of the dequantising kernels (all zero: Eq. 11 as is, dense y).
  int64_t beta_rows;                               // output features per beta block (0: one block);
                                                   // beta is [N/beta_rows, G], rowsum stays [N, G]
  int relu;                                        // y = max(y, 0) before the residual
  const void* residual; int64_t ld_res;            // y += residual[m, n] (dtype yt, row stride ld_res)
  int64_t ld_y;                                    // row stride of y in elements (0: N)
  uint32_t* status;                                // device status word (tensor-core path)
  int keep_status;                                 // the kernel before this one already cleared it
  void* scratch;                                   // gemm_tc_scratch_bytes(G) bytes (tensor-core path)
};
cudaError_t launch_gemm_simple(const GemmArgs& a, cudaStream_t s);
cudaError_t launch_gemm_tc(const GemmArgs& a, cudaStream_t s);      // tcgen05, two SMs per tile (gemm_tc2.cu)
bool gemm_tc_supported(int64_t M, int64_t K, int64_t N, int G);
size_t gemm_tc_scratch_bytes(int64_t M, int64_t N, int G);   // host-only, no device query

struct GemvArgs {
  const void* x; bl_dtype xt; int64_t K, N; int G; bl_quant_mode mode; float ln_eps;
  int eta_correction; const uint8_t* W_packed; const float* beta; const int32_t* rowsum;
  void* y; bl_dtype yt;
  uint32_t* clear_status = nullptr;   // when set: a status word that the call's (first) kernel clears, in stream order
};
cudaError_t launch_gemv_decode(const GemvArgs& a, cudaStream_t s);
cudaError_t gemv_decode_take_fallbacks(unsigned int* out);   // warps that read weights from global memory after a wait ran out
// The same for M tokens (x [M,K], y [M,N]) sharing one pass over the weights per 8 tokens.
cudaError_t launch_gemv_batch(const GemvArgs& a, int64_t M, cudaStream_t s);
bool gemv_batch_supported(int64_t M, int64_t K, int64_t N, int G);
cudaError_t launch_gemv_batch_pre(const GemvArgs& g, int64_t M, const int8_t* codes, const float* gamma, const int* csum,
                                  cudaStream_t s);   // the same kernel on tokens quantised earlier on the stream
// The same with a workspace: tokens quantised once by a kernel of their own, the product on the
// tcgen05 tensor cores, 16 tokens per pass over the weights (gemv_tc.cu).
cudaError_t launch_gemv_tc(const GemvArgs& a, int64_t M, void* ws, cudaStream_t s);
bool gemv_tc_supported(int64_t M, int64_t K, int64_t N, int G, int eta_correction);
size_t gemv_tc_ws_bytes(int64_t M, int64_t K);

// Decoder-block glue (fp16): the causal attention core.
cudaError_t launch_attention_causal(const void* q, const void* k, const void* v, void* o, int batch, int S,
                                    int heads, int64_t ld, int64_t ld_o, cudaStream_t s);

// Attention at inference (qk_norm_rope.cu, attention_window.cu, kv4_cache.cu, attention_kv4.cu).
struct NormRopeArgs {
  const void* q; const void* k; bl_dtype dt; int64_t T; int heads, kv_heads, head_dim; int64_t ld_q, ld_k;
  const void* wq; const void* wk; float eps; int rot_dim, interleaved; const float* inv_freq; const int32_t* positions;
  void* q_out; void* k_out; int64_t ld_qo, ld_ko;
};
cudaError_t launch_qk_norm_rope(const NormRopeArgs& a, cudaStream_t s);

struct WindowArgs {
  const void* q; const void* k; const void* v; void* o; bl_dtype dt; int batch; const int32_t* cu_q; const int32_t* cu_k;
  int64_t seq_q, seq_k, rows_q, rows_k; int heads, kv_heads, head_dim; int64_t ld_q, ld_k, ld_v, ld_o;
  int window, sinks; float scale;
};
cudaError_t launch_attention_window(const WindowArgs& a, cudaStream_t s);
cudaError_t window_take_fallbacks(unsigned int* out);       // CTAs that computed their rows the slow way after a wait ran out

cudaError_t launch_kv4_append(const bl_kv4_cache& c, const void* k, const void* v, int64_t T, int64_t ld_k, int64_t ld_v,
                              const int64_t* slots, cudaStream_t s);
cudaError_t launch_kv4_read(const bl_kv4_cache& c, void* k, void* v, int64_t T, int64_t ld_k, int64_t ld_v,
                            const int64_t* slots, cudaStream_t s);
cudaError_t launch_kv4_copy_pages(void* pages, size_t page_bytes, int64_t num_pages, int layers, size_t layer_stride,
                                  const int32_t* pairs, int64_t n, cudaStream_t s);

struct Kv4AttnArgs {
  const void* q; int batch, n_q, heads; int64_t ld_q; bl_kv4_cache cache; const int32_t* table; int64_t max_pages;
  const int32_t* lens; int window, sinks; float scale; void* o; int64_t ld_o; void* ws;
};
size_t attention_kv4_ws_bytes(int batch, int n_q, int heads, int kv_heads, int head_dim);
cudaError_t launch_attention_kv4(const Kv4AttnArgs& a, cudaStream_t s);

// 8-bit layers and experts (rms_norm_quant.cu, route_topk.cu, matmul.cu with matmul_narrow.cu and matmul_wide.cu).
struct NormQuantArgs {
  const void* x; bl_dtype dt; int64_t x_rows, T, K, ld_x; const int32_t* rows; const float* row_weights; int top_k;
  const void* residual; int64_t ld_res; const void* weight; float eps;
  void* h; int64_t ld_h; void* y; int64_t ld_y; int8_t* x_q; int64_t ld_q; float* scale; float inv_k;
};
cudaError_t launch_rms_norm_quant(const NormQuantArgs& a, cudaStream_t s);

struct RouteArgs {
  const void* logits; bl_dtype dt; int64_t T; int experts; int64_t ld; int top_k, normalise; const int32_t* positions;
  int32_t* chosen; float* weights; int32_t* offsets; int32_t* rows; int32_t* places;
  unsigned long long* members; uint8_t* counts; int32_t* sums; int stride;     // in the workspace, set by the launcher
};
size_t route_topk_ws_bytes(int64_t T, int experts);
cudaError_t launch_route_topk(RouteArgs a, void* ws, cudaStream_t s);

// y[r, n] = (sum_k x[source of r, k] w[expert of r, n, k]) x_scale w_scale + bias, ReLU, + residual.
struct MatmulArgs {
  bl_dtype operand;                                // BL_I8, BL_F16 or BL_BF16
  const void* x; int64_t x_rows, K, N, ld_x; const float* x_scale;
  const void* w; int64_t ld_w, expert_stride; const float* w_scale; int experts;
  const int32_t* offsets;                          // nullptr: one expert, every row
  const int32_t* rows; int64_t R;                  // rows of y
  const void* bias; int relu; const void* residual; int64_t ld_res;
  void* y; bl_dtype yt; int64_t ld_y;
};
cudaError_t launch_matmul(const MatmulArgs& a, cudaStream_t s);
cudaError_t launch_matmul_narrow(const MatmulArgs& a, int tokens, int splits, int per_sm, cudaStream_t s);   // tokens 16, 32 or 64
cudaError_t launch_matmul_wide(const MatmulArgs& a, int tile_rows, cudaStream_t s);              // 32..256, in steps of 32

// Host-side layout maps (also exported through bitlinear_layout_index).
int64_t prefill_bytes(int64_t N, int64_t K);
void prefill_index(int64_t K, int64_t n, int64_t k, int64_t* byte_off, int* bit);
void decode_index(int64_t K, int64_t n, int64_t k, int64_t* byte_off, int* bit);

}  // namespace bl
