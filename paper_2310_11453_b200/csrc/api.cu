// extern "C" entry points: argument validation on the host, workspace carving, launches.
// Nothing here allocates device memory or synchronises (bitlinear_ws_status excepted).
#include <math.h>

#include <initializer_list>
#include <utility>

#include "common.cuh"

namespace bl {
std::atomic<long long> g_debug_wait_polls{-1};
std::atomic<int> g_debug_meet_skew{0};
}  // namespace bl

namespace {

using namespace bl;

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline size_t round256(size_t v) { return (v + 255) & ~size_t(255); }
inline bool valid_dtype(int t) { return t == BL_F32 || t == BL_F16 || t == BL_BF16; }

// Common shape rules: sizes positive, 1 <= G <= BL_MAX_GROUPS, K % (8 G) == 0.
inline bl_status check_kg(int64_t K, int G) {
  if (K <= 0 || G < 1) return BL_ERR_SHAPE;
  if (G > BL_MAX_GROUPS) return BL_ERR_UNSUPPORTED;
  if (K % (8 * (int64_t)G) != 0) return BL_ERR_SHAPE;
  return BL_OK;
}

constexpr size_t kStatusBytes = 256;   // status word lives at the start of a GEMM workspace

// A GEMM workspace is the status word followed by the tensor-core kernel's scratch.
size_t gemm_ws_total(int64_t M, int64_t N, int G) {
  return kStatusBytes + round256(gemm_tc_scratch_bytes(M, N, G));
}

struct BlockWs {                       // carving of the BL_OP_BLOCK_FORWARD workspace
  size_t gemm, codes, gamma, eta, total;
};
BlockWs carve_block(int64_t T, int64_t d, int64_t ffn) {
  BlockWs w;
  size_t off = 0;
  const int64_t widest = ffn > 3 * d ? ffn : 3 * d;       // Q, K, V may run as one [3d, d] GEMM
  w.gemm = off;  off += gemm_ws_total(T, widest, 1);
  w.codes = off; off += round256((size_t)T * (size_t)widest);
  w.gamma = off; off += round256((size_t)T * sizeof(float));
  w.eta = off;   off += round256((size_t)T * sizeof(float));
  w.total = off;
  return w;
}

struct ForwardWs {                     // carving of the BL_OP_FORWARD workspace
  size_t status, codes, gamma, eta, quant, total;
};
ForwardWs carve_forward(int64_t M, int64_t N, int64_t K, int G) {
  ForwardWs w;
  size_t off = 0;
  w.status = off; off += gemm_ws_total(M, N, G);
  w.codes = off;  off += round256((size_t)M * (size_t)K);
  w.gamma = off;  off += round256((size_t)M * (size_t)G * sizeof(float));
  w.eta = off;    off += round256((size_t)M * (size_t)G * sizeof(float));
  w.quant = off;  off += round256(quant_ws_bytes(M, G));
  w.total = off;
  return w;
}

struct LatentWs {                      // carving of the BL_OP_FORWARD_LATENT workspace
  size_t pack, packed, alpha, beta, rowsum, forward, total;
  bl_layout layout;
};
LatentWs carve_latent(int64_t M, int64_t N, int64_t K, int G) {
  LatentWs w;
  w.layout = gemm_tc_supported(M, K, N, G) ? BL_LAYOUT_PREFILL : BL_LAYOUT_CANONICAL;
  size_t off = 0;
  w.pack = off;    off += round256(pack_ws_bytes(G));
  w.packed = off;  off += round256(w.layout == BL_LAYOUT_PREFILL ? (size_t)prefill_bytes(N, K) : (size_t)(N * (K / 8)));
  w.alpha = off;   off += round256((size_t)G * sizeof(float));
  w.beta = off;    off += round256((size_t)G * sizeof(float));
  w.rowsum = off;  off += round256((size_t)N * (size_t)G * sizeof(int32_t));
  w.forward = off; off += carve_forward(M, N, K, G).total;
  w.total = off;
  return w;
}

bl_status check_layout_for_gemm(bl_layout layout, int64_t M, int64_t K, int64_t N, int G) {
  if (layout == BL_LAYOUT_CANONICAL) return BL_OK;
  if (layout == BL_LAYOUT_PREFILL) return gemm_tc_supported(M, K, N, G) ? BL_OK : BL_ERR_SHAPE;
  return BL_ERR_UNSUPPORTED;
}

// ---- checks of the attention operators ---------------------------------------------------------
constexpr int kMaxHeads = 4096;
constexpr int64_t kMaxRows = 1 << 30;  // tokens: row numbers and positions stay inside 32 bits in the kernels

inline bool attention_dtype(int t) { return t == BL_F16 || t == BL_BF16; }
// 0: no window; one that no position can leave is none.
inline int clip_window(int window) { return window > 0 && window < kMaxRows ? window : 0; }
inline bool aligned_to(const void* p, unsigned n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
// The kernels multiply scores by scale . log2(e), which has to be finite.
inline bool score_scale(float scale) { return scale >= 0.f && scale <= 2.0e38f; }
// Query rows of attention_kv4: batch x n_q tokens of `heads` heads.
inline bool query_rows(int batch, int n_q, int heads) {
  return batch >= 0 && n_q >= 1 && heads >= 1 && heads <= kMaxHeads && (int64_t)batch * n_q <= kMaxRows &&
         (int64_t)batch * n_q * heads <= kMaxRows && (int64_t)n_q * heads <= kMaxRows;
}
// A row stride takes the row and keeps every row 16-byte aligned.
inline bool row_stride(int64_t ld, int heads, int head_dim) { return ld >= (int64_t)heads * head_dim && ld % 8 == 0; }

// ---- checks of the 8-bit layers ------------------------------------------------------------------
constexpr int kMaxRouted = 512, kMaxExperts = 1024;
constexpr int64_t kMaxStride = (int64_t)1 << 38;     // tensor maps take strides of up to 2^40 bytes
constexpr int64_t kMaxFeatures = 1 << 24;

// The sizes of a matrix product of R rows.
bl_status check_product(int operand, int64_t R, int64_t K, int64_t N, int64_t ld_x, int64_t ld_w, int64_t ld_y) {
  const int64_t unit = operand == BL_I8 ? 16 : 8;     // values in 16 bytes
  if (R < 0 || R > kMaxRows || N < 1 || N > kMaxFeatures) return BL_ERR_SHAPE;
  if (K < unit || K % unit != 0 || K > (operand == BL_I8 ? 131056 : 1 << 20)) return BL_ERR_SHAPE;
  if (ld_x < K || ld_x % unit != 0 || ld_x > kMaxStride || ld_w < K || ld_w % unit != 0 || ld_w > kMaxStride) return BL_ERR_SHAPE;
  return ld_y < N || ld_y > kMaxStride ? BL_ERR_SHAPE : BL_OK;
}

bl_status check_cache(const bl_kv4_cache* c) {
  if (!c) return BL_ERR_NULL;
  if (!attention_dtype(c->dtype) || (c->head_dim != 64 && c->head_dim != 128)) return BL_ERR_UNSUPPORTED;
  if (bitlinear_kv4_page_bytes(c->page_size, c->kv_heads, c->head_dim) == 0) return BL_ERR_SHAPE;
  if (c->num_pages < 0 || c->num_pages > 0x7FFFFFFF) return BL_ERR_SHAPE;
  if (c->num_pages > 0 && !c->pages) return BL_ERR_NULL;
  return aligned16(c->pages) ? BL_OK : BL_ERR_ALIGN;
}

}  // namespace

extern "C" {

const char* bitlinear_status_string(bl_status st) {
  switch (st) {
    case BL_OK: return "ok";
    case BL_ERR_NULL: return "null pointer";
    case BL_ERR_SHAPE: return "invalid shape";
    case BL_ERR_ALIGN: return "pointer not 16-byte aligned";
    case BL_ERR_UNSUPPORTED: return "unsupported option";
    case BL_ERR_WORKSPACE: return "workspace missing or too small";
    case BL_ERR_CUDA: return "CUDA runtime error";
    case BL_ERR_TIMEOUT: return "device-side wait timed out";
    case BL_ERR_TOO_LARGE: return "problem exceeds the built-in scratch of the no-allocation entry point";
  }
  return "unknown status";
}

size_t bitlinear_workspace_bytes(bl_op op, int64_t M, int64_t N, int64_t K, int G) {
  if (check_kg(K, G) != BL_OK) return 0;
  switch (op) {
    case BL_OP_BINARIZE_PACK: return round256(pack_ws_bytes(G));
    case BL_OP_QUANT_ACT: return M > 0 ? round256(quant_ws_bytes(M, G)) : 0;
    case BL_OP_FORWARD: return (M > 0 && N > 0) ? carve_forward(M, N, K, G).total : 0;
    case BL_OP_MATMUL_I32:
    case BL_OP_MATMUL_DEQUANT: return (M > 0 && N > 0) ? gemm_ws_total(M, N, G) : 0;
    case BL_OP_BLOCK_FORWARD: return (M > 0 && N > 0) ? carve_block(M, K, N).total : 0;
    case BL_OP_FORWARD_LATENT: return (M > 0 && N > 0) ? carve_latent(M, N, K, G).total : 0;
    case BL_OP_GEMV_DECODE_BATCH: return M > 0 ? round256(gemv_tc_ws_bytes(M, K)) : 0;
  }
  return 0;
}

size_t bitlinear_packed_bytes(bl_layout layout, int64_t N, int64_t K) {
  if (N <= 0 || K <= 0 || K % 8 != 0) return 0;
  switch (layout) {
    case BL_LAYOUT_CANONICAL: return (size_t)(N * (K / 8));
    case BL_LAYOUT_PREFILL: return K % 16 == 0 ? (size_t)prefill_bytes(N, K) : 0;
    case BL_LAYOUT_DECODE: return (K % 256 == 0 && N % 16 == 0) ? (size_t)(N * (K / 8)) : 0;
  }
  return 0;
}

bl_status bitlinear_layout_index(bl_layout layout, int64_t N, int64_t K, int64_t n, int64_t k,
                                 int64_t* byte_offset, int* bit) {
  if (!byte_offset || !bit) return BL_ERR_NULL;
  if (bitlinear_packed_bytes(layout, N, K) == 0 || n < 0 || n >= N || k < 0 || k >= K)
    return BL_ERR_SHAPE;
  switch (layout) {
    case BL_LAYOUT_CANONICAL: *byte_offset = n * (K / 8) + k / 8; *bit = (int)(k % 8); break;
    case BL_LAYOUT_PREFILL: prefill_index(K, n, k, byte_offset, bit); break;
    case BL_LAYOUT_DECODE: decode_index(K, n, k, byte_offset, bit); break;
  }
  return BL_OK;
}

bl_status bitlinear_binarize_pack(const void* W, bl_dtype wt, int64_t N, int64_t K, int G,
                                  bl_layout layout, const float* alpha_in, uint8_t* W_packed,
                                  float* alpha, float* beta, int32_t* rowsum, void* ws,
                                  size_t ws_bytes, void* stream) {
  if (!W || !W_packed || !alpha || !beta) return BL_ERR_NULL;
  if (N <= 0) return BL_ERR_SHAPE;
  bl_status st = check_kg(K, G);
  if (st != BL_OK) return st;
  if (!valid_dtype(wt)) return BL_ERR_UNSUPPORTED;
  if (layout != BL_LAYOUT_CANONICAL && layout != BL_LAYOUT_PREFILL && layout != BL_LAYOUT_DECODE)
    return BL_ERR_UNSUPPORTED;
  if (bitlinear_packed_bytes(layout, N, K) == 0) return BL_ERR_SHAPE;
  if (layout == BL_LAYOUT_PREFILL && (K / G) % 128 != 0) return BL_ERR_SHAPE;
  if (!aligned16(W) || !aligned16(W_packed)) return BL_ERR_ALIGN;
  if (!ws || ws_bytes < bitlinear_workspace_bytes(BL_OP_BINARIZE_PACK, 1, N, K, G)) return BL_ERR_WORKSPACE;
  if (!aligned16(ws)) return BL_ERR_ALIGN;
  PackArgs a{W, wt, N, K, G, layout, alpha_in, W_packed, alpha, beta, rowsum, ws};
  return launch_binarize_pack(a, (cudaStream_t)stream) == cudaSuccess ? BL_OK : BL_ERR_CUDA;
}

bl_status bitlinear_quant_act(const void* x, bl_dtype xt, int64_t M, int64_t K, int G, int b,
                              bl_quant_mode mode, bl_gran gran, float ln_eps, int8_t* x_q,
                              float* gamma, float* eta, void* ws, size_t ws_bytes, void* stream) {
  if (!x || !x_q || !gamma) return BL_ERR_NULL;
  if (mode == BL_ETA && !eta) return BL_ERR_NULL;
  if (M <= 0) return BL_ERR_SHAPE;
  bl_status st = check_kg(K, G);
  if (st != BL_OK) return st;
  if (b != 8 || !valid_dtype(xt)) return BL_ERR_UNSUPPORTED;
  if (mode != BL_ABSMAX && mode != BL_ETA) return BL_ERR_UNSUPPORTED;
  if (gran != BL_PER_TENSOR && gran != BL_PER_TOKEN) return BL_ERR_UNSUPPORTED;
  if ((K / G) * sizeof(float) > 200 * 1024) return BL_ERR_SHAPE;   // one segment must fit in shared memory
  if (M * (int64_t)G > 0x7FFFFFFF) return BL_ERR_SHAPE;
  if (!aligned16(x) || !aligned16(x_q)) return BL_ERR_ALIGN;
  if (gran == BL_PER_TENSOR) {
    if (!ws || ws_bytes < bitlinear_workspace_bytes(BL_OP_QUANT_ACT, M, 1, K, G)) return BL_ERR_WORKSPACE;
    if (!aligned16(ws)) return BL_ERR_ALIGN;
  }
  QuantArgs a{x, xt, M, K, G, mode, gran, ln_eps, x_q, gamma, eta, ws};
  // per-token scope needs no workspace; given one, its first word serves as the status word and the
  // kernel may then use copies whose wait is bounded and reported there
  if (gran == BL_PER_TOKEN && ws && ws_bytes >= kStatusBytes && aligned16(ws)) a.status = reinterpret_cast<uint32_t*>(ws);
  return launch_quant_act(a, (cudaStream_t)stream) == cudaSuccess ? BL_OK : BL_ERR_CUDA;
}

bl_status bitlinear_matmul_i32(const int8_t* x_q, int64_t M, int64_t K, int64_t N, int G,
                               const uint8_t* W_packed, bl_layout layout, int32_t* acc, void* ws,
                               size_t ws_bytes, void* stream) {
  if (!x_q || !W_packed || !acc) return BL_ERR_NULL;
  if (M <= 0 || N <= 0) return BL_ERR_SHAPE;
  bl_status st = check_kg(K, G);
  if (st != BL_OK) return st;
  st = check_layout_for_gemm(layout, M, K, N, G);
  if (st != BL_OK) return st;
  if (!aligned16(x_q) || !aligned16(W_packed) || !aligned16(acc)) return BL_ERR_ALIGN;
  if (!ws || ws_bytes < gemm_ws_total(M, N, G)) return BL_ERR_WORKSPACE;
  if (!aligned16(ws)) return BL_ERR_ALIGN;
  cudaStream_t s = (cudaStream_t)stream;
  // the tensor-core kernel clears the status word itself; the CUDA-core kernel never writes it
  if (layout != BL_LAYOUT_PREFILL && cudaMemsetAsync(ws, 0, kStatusBytes, s) != cudaSuccess) return BL_ERR_CUDA;
  GemmArgs a{};
  a.x_q = x_q; a.M = M; a.K = K; a.N = N; a.G = G; a.W_packed = W_packed; a.acc = acc;
  a.y = nullptr; a.gran = BL_PER_TENSOR; a.status = reinterpret_cast<uint32_t*>(ws);
  a.scratch = reinterpret_cast<char*>(ws) + kStatusBytes;
  cudaError_t e = (layout == BL_LAYOUT_PREFILL) ? launch_gemm_tc(a, s) : launch_gemm_simple(a, s);
  return e == cudaSuccess ? BL_OK : BL_ERR_CUDA;
}

bl_status bitlinear_matmul_dequant_ex(const int8_t* x_q, int64_t M, int64_t K, int64_t N, int G,
                                      bl_gran gran, const float* gamma, const float* eta,
                                      int eta_correction, const uint8_t* W_packed, bl_layout layout,
                                      const float* beta, const int32_t* rowsum, const bl_epilogue* epi,
                                      void* y, bl_dtype yt, void* ws, size_t ws_bytes, void* stream) {
  if (!x_q || !W_packed || !beta || !gamma || !y) return BL_ERR_NULL;
  if (eta_correction && (!rowsum || !eta)) return BL_ERR_NULL;
  if (M <= 0 || N <= 0) return BL_ERR_SHAPE;
  bl_status st = check_kg(K, G);
  if (st != BL_OK) return st;
  if (!valid_dtype(yt)) return BL_ERR_UNSUPPORTED;
  if (gran != BL_PER_TENSOR && gran != BL_PER_TOKEN) return BL_ERR_UNSUPPORTED;
  st = check_layout_for_gemm(layout, M, K, N, G);
  if (st != BL_OK) return st;
  bl_epilogue o{};
  if (epi) o = *epi;
  if (o.beta_rows < 0 || (o.beta_rows > 0 && (N % o.beta_rows != 0 || o.beta_rows % 32 != 0))) return BL_ERR_SHAPE;
  if (o.ld_y < 0 || (o.ld_y > 0 && o.ld_y < N)) return BL_ERR_SHAPE;
  if (o.residual && o.ld_res < N) return BL_ERR_SHAPE;
  if (!aligned16(x_q) || !aligned16(W_packed) || !aligned16(y) || !aligned16(o.residual)) return BL_ERR_ALIGN;
  if (!ws || ws_bytes < gemm_ws_total(M, N, G)) return BL_ERR_WORKSPACE;
  if (!aligned16(ws)) return BL_ERR_ALIGN;
  cudaStream_t s = (cudaStream_t)stream;
  // the tensor-core kernel clears the status word itself; the CUDA-core kernel never writes it
  if (layout != BL_LAYOUT_PREFILL && cudaMemsetAsync(ws, 0, kStatusBytes, s) != cudaSuccess) return BL_ERR_CUDA;
  GemmArgs a{};
  a.x_q = x_q; a.M = M; a.K = K; a.N = N; a.G = G; a.W_packed = W_packed; a.acc = nullptr;
  a.y = y; a.yt = yt; a.beta = beta; a.gamma = gamma; a.eta = eta; a.gran = gran;
  a.rowsum = rowsum; a.eta_correction = eta_correction ? 1 : 0;
  a.beta_rows = o.beta_rows; a.relu = o.relu ? 1 : 0; a.residual = o.residual; a.ld_res = o.ld_res; a.ld_y = o.ld_y;
  a.status = reinterpret_cast<uint32_t*>(ws);
  a.scratch = reinterpret_cast<char*>(ws) + kStatusBytes;
  cudaError_t e = (layout == BL_LAYOUT_PREFILL) ? launch_gemm_tc(a, s) : launch_gemm_simple(a, s);
  return e == cudaSuccess ? BL_OK : BL_ERR_CUDA;
}

bl_status bitlinear_matmul_dequant(const int8_t* x_q, int64_t M, int64_t K, int64_t N, int G,
                                   bl_gran gran, const float* gamma, const float* eta,
                                   int eta_correction, const uint8_t* W_packed, bl_layout layout,
                                   const float* beta, const int32_t* rowsum, void* y, bl_dtype yt,
                                   void* ws, size_t ws_bytes, void* stream) {
  return bitlinear_matmul_dequant_ex(x_q, M, K, N, G, gran, gamma, eta, eta_correction, W_packed, layout, beta,
                                     rowsum, nullptr, y, yt, ws, ws_bytes, stream);
}

bl_status bitlinear_binarize_pack_nsplit(const void* W, bl_dtype wt, int64_t N, int64_t K, int G, int NB,
                                         bl_layout layout, const float* alpha_in, uint8_t* W_packed,
                                         float* alpha, float* beta, int32_t* rowsum, void* ws,
                                         size_t ws_bytes, void* stream) {
  if (NB <= 0 || N <= 0 || N % NB != 0) return BL_ERR_SHAPE;
  if (!valid_dtype(wt)) return BL_ERR_UNSUPPORTED;
  const int64_t rows = N / NB;
  if (layout == BL_LAYOUT_PREFILL && NB > 1 && rows % 128 != 0) return BL_ERR_SHAPE;
  const size_t block_bytes = bitlinear_packed_bytes(layout, rows, K);
  if (block_bytes == 0) return BL_ERR_SHAPE;
  const size_t esz = wt == BL_F32 ? 4 : 2;
  for (int j = 0; j < NB; ++j) {
    const bl_status st = bitlinear_binarize_pack(
        reinterpret_cast<const char*>(W) + (size_t)j * (size_t)rows * (size_t)K * esz, wt, rows, K, G, layout,
        alpha_in ? alpha_in + (size_t)j * G : nullptr, W_packed ? W_packed + (size_t)j * block_bytes : nullptr,
        alpha ? alpha + (size_t)j * G : nullptr, beta ? beta + (size_t)j * G : nullptr,
        rowsum ? rowsum + (size_t)j * (size_t)rows * G : nullptr, ws, ws_bytes, stream);
    if (st != BL_OK) return st;
  }
  return BL_OK;
}

bl_status bitlinear_forward(const void* x, bl_dtype xt, int64_t M, int64_t K, int64_t N, int G,
                            int b, bl_quant_mode mode, bl_gran gran, float ln_eps,
                            int eta_correction, const uint8_t* W_packed, bl_layout layout,
                            const float* beta, const int32_t* rowsum, void* y, bl_dtype yt,
                            void* ws, size_t ws_bytes, void* stream) {
  if (!x || !W_packed || !beta || !y) return BL_ERR_NULL;
  if (eta_correction && !rowsum) return BL_ERR_NULL;
  if (M <= 0 || N <= 0) return BL_ERR_SHAPE;
  bl_status st = check_kg(K, G);
  if (st != BL_OK) return st;
  if (b != 8 || !valid_dtype(xt) || !valid_dtype(yt)) return BL_ERR_UNSUPPORTED;
  if (mode != BL_ABSMAX && mode != BL_ETA) return BL_ERR_UNSUPPORTED;
  if (gran != BL_PER_TENSOR && gran != BL_PER_TOKEN) return BL_ERR_UNSUPPORTED;
  if (eta_correction && mode != BL_ETA) return BL_ERR_UNSUPPORTED;
  st = check_layout_for_gemm(layout, M, K, N, G);
  if (st != BL_OK) return st;
  if ((K / G) * sizeof(float) > 200 * 1024 || M * (int64_t)G > 0x7FFFFFFF) return BL_ERR_SHAPE;
  if (!aligned16(x) || !aligned16(W_packed) || !aligned16(y)) return BL_ERR_ALIGN;
  const ForwardWs w = carve_forward(M, N, K, G);
  if (!ws || ws_bytes < w.total) return BL_ERR_WORKSPACE;
  if (!aligned16(ws)) return BL_ERR_ALIGN;
  char* base = reinterpret_cast<char*>(ws);
  cudaStream_t s = (cudaStream_t)stream;
  if (layout != BL_LAYOUT_PREFILL && cudaMemsetAsync(base + w.status, 0, kStatusBytes, s) != cudaSuccess)
    return BL_ERR_CUDA;
  int8_t* codes = reinterpret_cast<int8_t*>(base + w.codes);
  float* gamma = reinterpret_cast<float*>(base + w.gamma);
  float* eta = reinterpret_cast<float*>(base + w.eta);
  QuantArgs q{x, xt, M, K, G, mode, gran, ln_eps, codes, gamma, eta, base + w.quant};
  // One status word for the call: the quant kernels clear it (and may report a timeout of their
  // own), so the GEMM that follows must not clear it again.
  q.status = reinterpret_cast<uint32_t*>(base + w.status);
  if (launch_quant_act(q, s) != cudaSuccess) return BL_ERR_CUDA;
  GemmArgs a{};
  a.keep_status = 1;
  a.x_q = codes; a.M = M; a.K = K; a.N = N; a.G = G; a.W_packed = W_packed; a.acc = nullptr;
  a.y = y; a.yt = yt; a.beta = beta; a.gamma = gamma; a.eta = eta; a.gran = gran;
  a.rowsum = rowsum; a.eta_correction = eta_correction ? 1 : 0;
  a.status = reinterpret_cast<uint32_t*>(base + w.status);
  a.scratch = base + w.status + kStatusBytes;
  cudaError_t e = (layout == BL_LAYOUT_PREFILL) ? launch_gemm_tc(a, s) : launch_gemm_simple(a, s);
  return e == cudaSuccess ? BL_OK : BL_ERR_CUDA;
}

bl_status bitlinear_forward_latent(const void* x, bl_dtype xt, const void* W, bl_dtype wt, int64_t M, int64_t K,
                                   int64_t N, int G, int b, bl_quant_mode mode, bl_gran gran, float ln_eps,
                                   int eta_correction, float* alpha_out, float* beta_out, void* y, bl_dtype yt,
                                   void* ws, size_t ws_bytes, void* stream) {
  if (!x || !W || !y) return BL_ERR_NULL;
  if (M <= 0 || N <= 0) return BL_ERR_SHAPE;
  bl_status st = check_kg(K, G);
  if (st != BL_OK) return st;
  const LatentWs c = carve_latent(M, N, K, G);
  if (!ws || ws_bytes < c.total) return BL_ERR_WORKSPACE;
  if (!aligned16(ws)) return BL_ERR_ALIGN;
  char* base = reinterpret_cast<char*>(ws);
  uint8_t* packed = reinterpret_cast<uint8_t*>(base + c.packed);
  float* alpha = reinterpret_cast<float*>(base + c.alpha);
  float* beta = reinterpret_cast<float*>(base + c.beta);
  int32_t* rowsum = reinterpret_cast<int32_t*>(base + c.rowsum);
  st = bitlinear_binarize_pack(W, wt, N, K, G, c.layout, nullptr, packed, alpha, beta, rowsum, base + c.pack,
                               round256(pack_ws_bytes(G)), stream);
  if (st != BL_OK) return st;
  cudaStream_t s = (cudaStream_t)stream;
  if (alpha_out && cudaMemcpyAsync(alpha_out, alpha, (size_t)G * sizeof(float), cudaMemcpyDeviceToDevice, s) != cudaSuccess)
    return BL_ERR_CUDA;
  if (beta_out && cudaMemcpyAsync(beta_out, beta, (size_t)G * sizeof(float), cudaMemcpyDeviceToDevice, s) != cudaSuccess)
    return BL_ERR_CUDA;
  return bitlinear_forward(x, xt, M, K, N, G, b, mode, gran, ln_eps, eta_correction, packed, c.layout, beta, rowsum, y,
                           yt, base + c.forward, c.total - c.forward, stream);
}

bl_status bitlinear_gemv_decode(const void* x, bl_dtype xt, int64_t K, int64_t N, int G, int b,
                                bl_quant_mode mode, float ln_eps, int eta_correction,
                                const uint8_t* W_packed, const float* beta,
                                const int32_t* rowsum, void* y, bl_dtype yt, void* stream) {
  if (!x || !W_packed || !beta || !y) return BL_ERR_NULL;
  if (eta_correction && !rowsum) return BL_ERR_NULL;
  if (N <= 0) return BL_ERR_SHAPE;
  bl_status st = check_kg(K, G);
  if (st != BL_OK) return st;
  if (b != 8 || !valid_dtype(xt) || !valid_dtype(yt)) return BL_ERR_UNSUPPORTED;
  if (mode != BL_ABSMAX && mode != BL_ETA) return BL_ERR_UNSUPPORTED;
  if (eta_correction && mode != BL_ETA) return BL_ERR_UNSUPPORTED;
  if (K % 256 != 0 || N % 16 != 0 || K > 32768) return BL_ERR_SHAPE;
  if (G > 1 && (K / G) % 128 != 0) return BL_ERR_SHAPE;
  if (!aligned16(x) || !aligned16(W_packed) || !aligned16(y)) return BL_ERR_ALIGN;
  GemvArgs a{x, xt, K, N, G, mode, ln_eps, eta_correction ? 1 : 0, W_packed, beta, rowsum, y, yt};
  return launch_gemv_decode(a, (cudaStream_t)stream) == cudaSuccess ? BL_OK : BL_ERR_CUDA;
}

bl_status bitlinear_gemv_decode_batch(const void* x, bl_dtype xt, int64_t M, int64_t K, int64_t N, int G,
                                      int b, bl_quant_mode mode, float ln_eps, int eta_correction,
                                      const uint8_t* W_packed, const float* beta, const int32_t* rowsum,
                                      void* y, bl_dtype yt, void* stream) {
  if (!x || !W_packed || !beta || !y) return BL_ERR_NULL;
  if (eta_correction && !rowsum) return BL_ERR_NULL;
  if (M <= 0 || N <= 0) return BL_ERR_SHAPE;
  bl_status st = check_kg(K, G);
  if (st != BL_OK) return st;
  if (b != 8 || !valid_dtype(xt) || !valid_dtype(yt)) return BL_ERR_UNSUPPORTED;
  if (mode != BL_ABSMAX && mode != BL_ETA) return BL_ERR_UNSUPPORTED;
  if (eta_correction && mode != BL_ETA) return BL_ERR_UNSUPPORTED;
  if (!gemv_batch_supported(M, K, N, G)) return BL_ERR_SHAPE;
  if (!aligned16(x) || !aligned16(W_packed) || !aligned16(y)) return BL_ERR_ALIGN;
  GemvArgs a{x, xt, K, N, G, mode, ln_eps, eta_correction ? 1 : 0, W_packed, beta, rowsum, y, yt};
  return launch_gemv_batch(a, M, (cudaStream_t)stream) == cudaSuccess ? BL_OK : BL_ERR_CUDA;
}

bl_status bitlinear_gemv_decode_batch_ws(const void* x, bl_dtype xt, int64_t M, int64_t K, int64_t N, int G,
                                         int b, bl_quant_mode mode, float ln_eps, int eta_correction,
                                         const uint8_t* W_packed, const float* beta, const int32_t* rowsum,
                                         void* y, bl_dtype yt, void* ws, size_t ws_bytes, void* stream) {
  if (!x || !W_packed || !beta || !y) return BL_ERR_NULL;
  if (eta_correction && !rowsum) return BL_ERR_NULL;
  if (M <= 0 || N <= 0) return BL_ERR_SHAPE;
  bl_status st = check_kg(K, G);
  if (st != BL_OK) return st;
  if (b != 8 || !valid_dtype(xt) || !valid_dtype(yt)) return BL_ERR_UNSUPPORTED;
  if (mode != BL_ABSMAX && mode != BL_ETA) return BL_ERR_UNSUPPORTED;
  if (eta_correction && mode != BL_ETA) return BL_ERR_UNSUPPORTED;
  if (!aligned16(x) || !aligned16(W_packed) || !aligned16(y)) return BL_ERR_ALIGN;
  GemvArgs a{x, xt, K, N, G, mode, ln_eps, eta_correction ? 1 : 0, W_packed, beta, rowsum, y, yt};
  if (gemv_tc_supported(M, K, N, G, eta_correction)) {
    if (!ws || ws_bytes < bitlinear_workspace_bytes(BL_OP_GEMV_DECODE_BATCH, M, N, K, G)) return BL_ERR_WORKSPACE;
    if (!aligned16(ws)) return BL_ERR_ALIGN;
    return launch_gemv_tc(a, M, ws, (cudaStream_t)stream) == cudaSuccess ? BL_OK : BL_ERR_CUDA;
  }
  // shapes the tensor-core form does not take: the kernel of bitlinear_gemv_decode_batch; of the workspace
  // only the status word is touched (cleared, so that bitlinear_ws_status answers for this call too)
  if (ws && ws_bytes >= sizeof(uint32_t) && aligned16(ws)) a.clear_status = reinterpret_cast<uint32_t*>(ws);
  if (!gemv_batch_supported(M, K, N, G)) return BL_ERR_SHAPE;
  return launch_gemv_batch(a, M, (cudaStream_t)stream) == cudaSuccess ? BL_OK : BL_ERR_CUDA;
}

bl_status bitlinear_attention_causal(const void* q, const void* k, const void* v, void* o, int batch, int seq,
                                     int heads, int head_dim, int64_t ld, int64_t ld_o, void* stream) {
  if (!q || !k || !v || !o) return BL_ERR_NULL;
  if (batch <= 0 || seq <= 0 || heads <= 0 || seq % 64 != 0 || ld % 8 != 0 || ld_o % 8 != 0) return BL_ERR_SHAPE;
  if (ld < (int64_t)heads * 128 || ld_o < (int64_t)heads * 128) return BL_ERR_SHAPE;
  if (head_dim != 128) return BL_ERR_UNSUPPORTED;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(o)) return BL_ERR_ALIGN;
  return launch_attention_causal(q, k, v, o, batch, seq, heads, ld, ld_o, (cudaStream_t)stream) == cudaSuccess
             ? BL_OK : BL_ERR_CUDA;
}

bl_status bitlinear_block_forward(const void* x, int batch, int seq, int heads, int64_t ffn, float ln_eps,
                                  const bl_block_weights* w, const bl_block_buffers* buf, void* y, void* ws,
                                  size_t ws_bytes, void* stream) {
  if (!x || !w || !buf || !y) return BL_ERR_NULL;
  if (!w->W_q || !w->W_k || !w->W_v || !w->W_o || !w->W_up || !w->W_down) return BL_ERR_NULL;
  if (!w->beta_q || !w->beta_k || !w->beta_v || !w->beta_o || !w->beta_up || !w->beta_down) return BL_ERR_NULL;
  if (!buf->q || !buf->k || !buf->v || !buf->a || !buf->h || !buf->u) return BL_ERR_NULL;
  if (batch <= 0 || seq <= 0 || heads <= 0 || ffn <= 0 || seq % 64 != 0 || ffn % 128 != 0) return BL_ERR_SHAPE;
  const int64_t T = (int64_t)batch * seq, d = (int64_t)heads * 128;
  if (!gemm_tc_supported(T, d, d, 1) || !gemm_tc_supported(T, d, ffn, 1) || !gemm_tc_supported(T, ffn, d, 1))
    return BL_ERR_SHAPE;
  const void* ptrs[] = {x, y, buf->q, buf->k, buf->v, buf->a, buf->h, buf->u, w->W_q, w->W_k, w->W_v, w->W_o,
                        w->W_up, w->W_down};
  for (const void* p : ptrs) if (!aligned16(p)) return BL_ERR_ALIGN;
  const int64_t ld_qkv = buf->ld_qkv > 0 ? buf->ld_qkv : d;
  if (ld_qkv < d || ld_qkv % 8 != 0) return BL_ERR_SHAPE;
  const BlockWs c = carve_block(T, d, ffn);
  if (!ws || ws_bytes < c.total) return BL_ERR_WORKSPACE;
  if (!aligned16(ws)) return BL_ERR_ALIGN;
  char* base = reinterpret_cast<char*>(ws);
  cudaStream_t s = (cudaStream_t)stream;
  int8_t* codes = reinterpret_cast<int8_t*>(base + c.codes);
  float* gamma = reinterpret_cast<float*>(base + c.gamma);
  float* eta = reinterpret_cast<float*>(base + c.eta);

  // LN + per-token quantisation of `in` [T,K] (fp16), then W~ x~ rescaled into `out` [T,N] (fp16).
  // One status word for the whole block: the first kernel clears it, every later one keeps it.
  uint32_t* status = reinterpret_cast<uint32_t*>(base + c.gemm);
  bool first_kernel = true;
  auto quant = [&](const void* in, int64_t K, bl_quant_mode mode) -> bool {
    QuantArgs q{in, BL_F16, T, K, 1, mode, BL_PER_TOKEN, ln_eps, codes, gamma, eta, nullptr};
    q.status = status;
    q.keep_status = first_kernel ? 0 : 1;
    first_kernel = false;
    return launch_quant_act(q, s) == cudaSuccess;
  };
  // out [T,N] (row stride ld) = [relu] BitLinear(codes) [+ res]; beta holds one entry per beta_rows features.
  auto matmul = [&](int64_t K, int64_t N, const uint8_t* W, const float* beta, int64_t beta_rows, void* out,
                    int64_t ld, bool relu, const void* res) -> bool {
    GemmArgs g{};
    g.x_q = codes; g.M = T; g.K = K; g.N = N; g.G = 1; g.W_packed = W; g.acc = nullptr; g.y = out; g.yt = BL_F16;
    g.beta = beta; g.gamma = gamma; g.eta = eta; g.gran = BL_PER_TOKEN; g.rowsum = nullptr; g.eta_correction = 0;
    g.beta_rows = beta_rows; g.relu = relu ? 1 : 0; g.residual = res; g.ld_res = d; g.ld_y = ld;
    g.status = status; g.keep_status = 1;
    g.scratch = base + c.gemm + kStatusBytes;
    return launch_gemm_tc(g, s) == cudaSuccess;
  };
  // Q, K, V as one GEMM when the caller laid them out for it: the three packed matrices and their
  // betas back to back (one [3d, d] matrix with a beta per d rows) and q, k, v as the column
  // blocks of one [T, 3d] buffer.
  const size_t wbytes = (size_t)prefill_bytes(d, d);
  const __half* qh = reinterpret_cast<const __half*>(buf->q);
  const bool fused_qkv = ld_qkv == 3 * d && w->W_k == w->W_q + wbytes && w->W_v == w->W_k + wbytes &&
                         w->beta_k == w->beta_q + 1 && w->beta_v == w->beta_k + 1 &&
                         buf->k == (const void*)(qh + d) && buf->v == (const void*)(qh + 2 * d);
  bool ok = quant(x, d, BL_ABSMAX);
  if (fused_qkv) {
    ok = ok && matmul(d, 3 * d, w->W_q, w->beta_q, d, buf->q, ld_qkv, false, nullptr);
  } else {
    ok = ok && matmul(d, d, w->W_q, w->beta_q, 0, buf->q, ld_qkv, false, nullptr)
            && matmul(d, d, w->W_k, w->beta_k, 0, buf->k, ld_qkv, false, nullptr)
            && matmul(d, d, w->W_v, w->beta_v, 0, buf->v, ld_qkv, false, nullptr);
  }
  ok = ok && launch_attention_causal(buf->q, buf->k, buf->v, buf->a, batch, seq, heads, ld_qkv, d, s) == cudaSuccess
      && quant(buf->a, d, BL_ABSMAX) && matmul(d, d, w->W_o, w->beta_o, 0, buf->h, d, false, x)
      && quant(buf->h, d, BL_ABSMAX) && matmul(d, ffn, w->W_up, w->beta_up, 0, buf->u, ffn, true, nullptr)
      && quant(buf->u, ffn, BL_ETA) && matmul(ffn, d, w->W_down, w->beta_down, 0, y, d, false, buf->h);
  return ok ? BL_OK : BL_ERR_CUDA;
}

bl_status bitlinear_qk_norm_rope(const void* q, const void* k, bl_dtype dt, int64_t T, int heads, int kv_heads,
                                 int head_dim, int64_t ld_q, int64_t ld_k, const void* wq, const void* wk,
                                 float eps, int rot_dim, int interleaved, const float* inv_freq,
                                 const int32_t* positions, void* q_out, void* k_out, int64_t ld_qo, int64_t ld_ko,
                                 void* stream) {
  if (!valid_dtype(dt)) return BL_ERR_UNSUPPORTED;
  if (T < 0 || T > kMaxRows || heads < 1 || kv_heads < 1 || heads > kMaxHeads || kv_heads > kMaxHeads) return BL_ERR_SHAPE;
  if (head_dim < 16 || head_dim > 256 || head_dim % 16 != 0) return BL_ERR_SHAPE;
  if (rot_dim < 0 || rot_dim > head_dim || rot_dim % 16 != 0 || eps != eps) return BL_ERR_SHAPE;
  if (!row_stride(ld_q, heads, head_dim) || !row_stride(ld_qo, heads, head_dim) || !row_stride(ld_k, kv_heads, head_dim) ||
      !row_stride(ld_ko, kv_heads, head_dim))
    return BL_ERR_SHAPE;
  if (T == 0) return BL_OK;
  if (!q || !k || !q_out || !k_out || !positions || (rot_dim > 0 && !inv_freq)) return BL_ERR_NULL;
  if (!aligned16(q) || !aligned16(k) || !aligned16(q_out) || !aligned16(k_out) || !aligned16(wq) || !aligned16(wk) ||
      !aligned_to(inv_freq, 4) || !aligned_to(positions, 4))
    return BL_ERR_ALIGN;
  if ((q == q_out && ld_q != ld_qo) || (k == k_out && ld_k != ld_ko)) return BL_ERR_SHAPE;
  NormRopeArgs a{q, k, dt, T, heads, kv_heads, head_dim, ld_q, ld_k, wq, wk, eps, rot_dim, interleaved ? 1 : 0, inv_freq,
                 positions, q_out, k_out, ld_qo, ld_ko};
  return launch_qk_norm_rope(a, (cudaStream_t)stream) == cudaSuccess ? BL_OK : BL_ERR_CUDA;
}

bl_status bitlinear_attention_window(const void* q, const void* k, const void* v, void* o, bl_dtype dt, int batch,
                                     const int32_t* cu_q, const int32_t* cu_k, int64_t seq_q, int64_t seq_k,
                                     int64_t rows_q, int64_t rows_k, int heads, int kv_heads, int head_dim,
                                     int64_t ld_q, int64_t ld_k, int64_t ld_v, int64_t ld_o, int window, int sinks,
                                     float scale, void* stream) {
  if (!attention_dtype(dt) || (head_dim != 64 && head_dim != 128)) return BL_ERR_UNSUPPORTED;
  if (batch < 0 || seq_q < 0 || seq_k < 0 || rows_q < 0 || rows_k < 0) return BL_ERR_SHAPE;
  if (seq_q > kMaxRows || seq_k > kMaxRows || rows_q > kMaxRows || rows_k > kMaxRows) return BL_ERR_SHAPE;
  if (heads < 1 || kv_heads < 1 || heads > kMaxHeads || heads % kv_heads != 0 || sinks < 0) return BL_ERR_SHAPE;
  if (!score_scale(scale)) return BL_ERR_SHAPE;
  if (cu_k && !cu_q) return BL_ERR_NULL;
  if (!cu_q && ((int64_t)batch * seq_q > rows_q || (int64_t)batch * seq_k > rows_k)) return BL_ERR_SHAPE;
  if (!row_stride(ld_q, heads, head_dim) || !row_stride(ld_o, heads, head_dim) || !row_stride(ld_k, kv_heads, head_dim) ||
      !row_stride(ld_v, kv_heads, head_dim))
    return BL_ERR_SHAPE;
  if (batch == 0 || seq_q == 0 || rows_q == 0) return BL_OK;
  if (!q || !o || (rows_k > 0 && (!k || !v))) return BL_ERR_NULL;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(o) || !aligned_to(cu_q, 4) || !aligned_to(cu_k, 4))
    return BL_ERR_ALIGN;
  int64_t blocks = (seq_q + 127) / 128 * batch;                  // blocks of query rows, at most
  if (cu_q && blocks > rows_q / 128 + batch) blocks = rows_q / 128 + batch;
  if (blocks * heads > 0x7FFFFFFF) return BL_ERR_SHAPE;
  WindowArgs a{q, k, v, o, dt, batch, cu_q, cu_k ? cu_k : cu_q, seq_q, seq_k, rows_q, rows_k, heads, kv_heads, head_dim, ld_q,
               ld_k, ld_v, ld_o, clip_window(window), sinks, scale};
  if (a.scale == 0.f) a.scale = 1.f / sqrtf((float)head_dim);
  return launch_attention_window(a, (cudaStream_t)stream) == cudaSuccess ? BL_OK : BL_ERR_CUDA;
}

size_t bitlinear_kv4_page_bytes(int page_size, int kv_heads, int head_dim) {
  if (page_size != 16 && page_size != 32 && page_size != 64) return 0;
  if (kv_heads < 1 || kv_heads > kMaxHeads || (head_dim != 64 && head_dim != 128)) return 0;
  return (size_t)page_size * (size_t)kv_heads * (size_t)(head_dim + 8);
}

bl_status bitlinear_kv4_append(const bl_kv4_cache* cache, const void* k, const void* v, int64_t T, int64_t ld_k,
                               int64_t ld_v, const int64_t* slots, void* stream) {
  const bl_status st = check_cache(cache);
  if (st != BL_OK) return st;
  if (T < 0 || T > kMaxRows || T * cache->kv_heads > 0x7FFFFFFF - 64) return BL_ERR_SHAPE;
  if (!row_stride(ld_k, cache->kv_heads, cache->head_dim) || !row_stride(ld_v, cache->kv_heads, cache->head_dim))
    return BL_ERR_SHAPE;
  if (T == 0) return BL_OK;
  if (!k || !v || !slots) return BL_ERR_NULL;
  if (!aligned16(k) || !aligned16(v) || !aligned_to(slots, 8)) return BL_ERR_ALIGN;
  return launch_kv4_append(*cache, k, v, T, ld_k, ld_v, slots, (cudaStream_t)stream) == cudaSuccess ? BL_OK : BL_ERR_CUDA;
}

bl_status bitlinear_kv4_read(const bl_kv4_cache* cache, void* k, void* v, int64_t T, int64_t ld_k, int64_t ld_v,
                             const int64_t* slots, void* stream) {
  const bl_status st = check_cache(cache);
  if (st != BL_OK) return st;
  if (T < 0 || T > kMaxRows || T * cache->kv_heads > 0x7FFFFFFF - 64) return BL_ERR_SHAPE;
  if (!row_stride(ld_k, cache->kv_heads, cache->head_dim) || !row_stride(ld_v, cache->kv_heads, cache->head_dim))
    return BL_ERR_SHAPE;
  if (T == 0) return BL_OK;
  if (!k || !v || !slots) return BL_ERR_NULL;
  if (!aligned16(k) || !aligned16(v) || !aligned_to(slots, 8)) return BL_ERR_ALIGN;
  return launch_kv4_read(*cache, k, v, T, ld_k, ld_v, slots, (cudaStream_t)stream) == cudaSuccess ? BL_OK : BL_ERR_CUDA;
}

size_t bitlinear_attention_kv4_ws_bytes(int batch, int n_q, int heads, int kv_heads, int head_dim) {
  if (!query_rows(batch, n_q, heads) || kv_heads < 1 || heads % kv_heads != 0) return 0;
  if (head_dim != 64 && head_dim != 128) return 0;
  return round256(attention_kv4_ws_bytes(batch, n_q, heads, kv_heads, head_dim));
}

bl_status bitlinear_attention_kv4(const void* q, int batch, int n_q, int heads, int64_t ld_q, const bl_kv4_cache* cache,
                                  const int32_t* block_table, int64_t max_pages, const int32_t* lens, int window,
                                  int sinks, float scale, void* o, int64_t ld_o, void* ws, size_t ws_bytes,
                                  void* stream) {
  const bl_status st = check_cache(cache);
  if (st != BL_OK) return st;
  if (!query_rows(batch, n_q, heads) || heads % cache->kv_heads != 0 || sinks < 0) return BL_ERR_SHAPE;
  if (max_pages < 0 || max_pages > kMaxRows / cache->page_size) return BL_ERR_SHAPE;
  if (!score_scale(scale)) return BL_ERR_SHAPE;
  if (!row_stride(ld_q, heads, cache->head_dim) || !row_stride(ld_o, heads, cache->head_dim)) return BL_ERR_SHAPE;
  if (batch == 0) return BL_OK;
  if (!q || !o || !lens || (max_pages > 0 && !block_table)) return BL_ERR_NULL;
  if (!aligned16(q) || !aligned16(o) || !aligned_to(block_table, 4) || !aligned_to(lens, 4)) return BL_ERR_ALIGN;
  const size_t need = bitlinear_attention_kv4_ws_bytes(batch, n_q, heads, cache->kv_heads, cache->head_dim);
  if (!ws || ws_bytes < need) return BL_ERR_WORKSPACE;
  if (!aligned16(ws)) return BL_ERR_ALIGN;
  Kv4AttnArgs a{q, batch, n_q, heads, ld_q, *cache, block_table, max_pages, lens, clip_window(window), sinks, scale, o, ld_o, ws};
  if (a.scale == 0.f) a.scale = 1.f / sqrtf((float)cache->head_dim);
  return launch_attention_kv4(a, (cudaStream_t)stream) == cudaSuccess ? BL_OK : BL_ERR_CUDA;
}

bl_status bitlinear_kv4_copy_pages(void* pages, size_t page_bytes, int64_t num_pages, int layers, size_t layer_stride,
                                   const int32_t* pairs, int64_t n, void* stream) {
  if (num_pages < 0 || num_pages > 0x7FFFFFFF || layers < 0 || n < 0 || n > 0x7FFFFFFF) return BL_ERR_SHAPE;
  if (page_bytes == 0 || page_bytes % 16 != 0) return BL_ERR_SHAPE;
  if (layers > 1 && (layer_stride % 16 != 0 || layer_stride / page_bytes < (size_t)num_pages)) return BL_ERR_SHAPE;
  if (layers > 65535 || page_bytes > ((size_t)1 << 40) || n * (int64_t)((page_bytes + 16383) / 16384) > 0x7FFFFFFF) return BL_ERR_SHAPE;
  if (n == 0 || layers == 0 || num_pages == 0) return BL_OK;
  if (!pages || !pairs) return BL_ERR_NULL;
  if (!aligned16(pages) || !aligned_to(pairs, 8)) return BL_ERR_ALIGN;
  return launch_kv4_copy_pages(pages, page_bytes, num_pages, layers, layers > 1 ? layer_stride : 0, pairs, n,
                               (cudaStream_t)stream) == cudaSuccess ? BL_OK : BL_ERR_CUDA;
}

bl_status bitlinear_rms_norm_quant(const void* x, bl_dtype dt, int64_t x_rows, int64_t T, int64_t K, int64_t ld_x,
                                   const int32_t* rows, const float* row_weights, int top_k, const void* residual,
                                   int64_t ld_res, const void* weight, float eps, void* h, int64_t ld_h, void* y,
                                   int64_t ld_y, int8_t* x_q, int64_t ld_q, float* scale, void* stream) {
  if (!valid_dtype(dt)) return BL_ERR_UNSUPPORTED;
  if (T < 0 || T > kMaxRows || x_rows < 0 || x_rows > kMaxRows || K < 8 || K > 32768 || K % 8 != 0 || eps != eps) return BL_ERR_SHAPE;
  if (rows ? (top_k < 1 || top_k > 64) : x_rows < T) return BL_ERR_SHAPE;
  if (row_weights && !rows) return BL_ERR_NULL;
  auto stride = [K](const void* p, int64_t ld) { return !p || (ld >= K && ld % 8 == 0 && ld <= kMaxStride); };
  if (ld_x < K || ld_x % 8 != 0 || ld_x > kMaxStride || !stride(residual, ld_res) || !stride(h, ld_h) || !stride(y, ld_y) || !stride(x_q, ld_q)) return BL_ERR_SHAPE;
  if (T == 0) return BL_OK;
  if ((!x && x_rows > 0) || (!h && !y && !x_q) || (x_q && !scale)) return BL_ERR_NULL;
  if (!aligned16(x) || !aligned16(residual) || !aligned16(weight) || !aligned16(h) || !aligned16(y) || !aligned_to(x_q, 8) ||
      !aligned_to(rows, 4) || !aligned_to(row_weights, 4) || !aligned_to(scale, 4))
    return BL_ERR_ALIGN;
  for (const auto& o : {std::make_pair((const void*)h, ld_h), std::make_pair((const void*)y, ld_y)})
    if (o.first && ((o.first == residual && o.second != ld_res) || (o.first == x && (rows || o.second != ld_x)))) return BL_ERR_SHAPE;
  NormQuantArgs a{x, dt, x_rows, T, K, ld_x, rows, row_weights, top_k, residual, ld_res, weight, eps, h, ld_h, y, ld_y, x_q, ld_q, scale, (float)(1.0 / (double)K)};
  return launch_rms_norm_quant(a, (cudaStream_t)stream) == cudaSuccess ? BL_OK : BL_ERR_CUDA;
}

bl_status bitlinear_matmul_i8(const int8_t* x_q, int64_t M, int64_t K, int64_t N, int64_t ld_x, const float* x_scale,
                              const int8_t* w_q, int64_t ld_w, const float* w_scale, const void* bias, int relu,
                              const void* residual, int64_t ld_res, void* y, bl_dtype yt, int64_t ld_y, void* stream) {
  if (!valid_dtype(yt)) return BL_ERR_UNSUPPORTED;
  const bl_status st = check_product(BL_I8, M, K, N, ld_x, ld_w, ld_y);
  if (st != BL_OK) return st;
  if (residual && (ld_res < N || ld_res > kMaxStride)) return BL_ERR_SHAPE;
  if (M == 0) return BL_OK;
  if (!x_q || !w_q || !y) return BL_ERR_NULL;
  const unsigned es = yt == BL_F32 ? 4 : 2;
  if (!aligned16(x_q) || !aligned16(w_q) || !aligned_to(y, es) || !aligned_to(bias, es) || !aligned_to(residual, es) ||
      !aligned_to(x_scale, 4) || !aligned_to(w_scale, 4))
    return BL_ERR_ALIGN;
  if (y == residual && ld_y != ld_res) return BL_ERR_SHAPE;
  MatmulArgs a{BL_I8, x_q, M, K, N, ld_x, x_scale, w_q, ld_w, 0, w_scale, 1, nullptr, nullptr, M, bias, relu ? 1 : 0, residual, ld_res, y, yt, ld_y};
  return launch_matmul(a, (cudaStream_t)stream) == cudaSuccess ? BL_OK : BL_ERR_CUDA;
}

size_t bitlinear_route_topk_ws_bytes(int64_t T, int experts) {
  if (T < 0 || T > kMaxRows || experts < 1 || experts > kMaxRouted) return 0;
  return round256(route_topk_ws_bytes(T, experts));
}

bl_status bitlinear_route_topk(const void* logits, bl_dtype dt, int64_t T, int experts, int64_t ld, int top_k,
                               int normalise, const int32_t* positions, int32_t* chosen, float* weights,
                               int32_t* offsets, int32_t* rows, int32_t* places, void* ws, size_t ws_bytes,
                               void* stream) {
  if (!valid_dtype(dt)) return BL_ERR_UNSUPPORTED;
  if (T < 0 || experts < 1 || experts > kMaxRouted || top_k < 1 || top_k > 32 || top_k > experts) return BL_ERR_SHAPE;
  if (T > kMaxRows / top_k || ld < experts || ld > kMaxStride) return BL_ERR_SHAPE;
  if (!offsets || (T > 0 && (!logits || !chosen || !weights || !rows || !places))) return BL_ERR_NULL;
  if (!aligned_to(logits, dt == BL_F32 ? 4 : 2) || !aligned_to(positions, 4) || !aligned_to(chosen, 4) || !aligned_to(weights, 4) ||
      !aligned_to(offsets, 4) || !aligned_to(rows, 4) || !aligned_to(places, 4))
    return BL_ERR_ALIGN;
  const size_t need = bitlinear_route_topk_ws_bytes(T, experts);
  if (need > 0 && (!ws || ws_bytes < need)) return BL_ERR_WORKSPACE;
  if (!aligned16(ws)) return BL_ERR_ALIGN;
  RouteArgs a{logits, dt, T, experts, ld, top_k, normalise ? 1 : 0, positions, chosen, weights, offsets, rows, places, nullptr, nullptr, nullptr, 0};
  return launch_route_topk(a, ws, (cudaStream_t)stream) == cudaSuccess ? BL_OK : BL_ERR_CUDA;
}

bl_status bitlinear_matmul_grouped(const void* x, bl_dtype operand, int64_t x_rows, int64_t K, int64_t N, int64_t ld_x,
                                   const float* x_scale, const void* w, int64_t ld_w, int64_t expert_stride,
                                   const float* w_scale, int experts, const int32_t* offsets, const int32_t* rows,
                                   int64_t R, const void* bias, int relu, void* y, bl_dtype yt, int64_t ld_y,
                                   void* stream) {
  if ((operand != BL_I8 && operand != BL_F16 && operand != BL_BF16) || !valid_dtype(yt)) return BL_ERR_UNSUPPORTED;
  if (operand != BL_I8 && (x_scale || w_scale)) return BL_ERR_UNSUPPORTED;
  const bl_status st = check_product(operand, R, K, N, ld_x, ld_w, ld_y);
  if (st != BL_OK) return st;
  if (experts < 1 || experts > kMaxExperts || x_rows < 0 || x_rows > kMaxRows || (rows ? x_rows < 1 && R > 0 : x_rows < R)) return BL_ERR_SHAPE;
  if (experts > 1 && (expert_stride % ld_w != 0 || expert_stride / ld_w < N || expert_stride > kMaxStride)) return BL_ERR_SHAPE;
  if (R == 0) return BL_OK;
  if (!x || !w || !offsets || !y) return BL_ERR_NULL;
  const unsigned es = yt == BL_F32 ? 4 : 2;
  if (!aligned16(x) || !aligned16(w) || !aligned_to(y, es) || !aligned_to(bias, es) || !aligned_to(x_scale, 4) ||
      !aligned_to(w_scale, 4) || !aligned_to(offsets, 4) || !aligned_to(rows, 4))
    return BL_ERR_ALIGN;
  MatmulArgs a{operand, x, x_rows, K, N, ld_x, x_scale, w, ld_w, expert_stride, w_scale, experts, offsets, rows, R, bias, relu ? 1 : 0,
               nullptr, 0, y, yt, ld_y};
  return launch_matmul(a, (cudaStream_t)stream) == cudaSuccess ? BL_OK : BL_ERR_CUDA;
}

bl_status bitlinear_ws_status(const void* ws, void* stream) {
  if (!ws) return BL_ERR_NULL;
  uint32_t word = 0;
  if (cudaStreamSynchronize((cudaStream_t)stream) != cudaSuccess) return BL_ERR_CUDA;
  if (cudaMemcpy(&word, ws, sizeof(word), cudaMemcpyDeviceToHost) != cudaSuccess) return BL_ERR_CUDA;
  const uint32_t n = word - kStatusPerWarp;            // words that follow
  if (n > kMostStatusWords) return word == 0 ? BL_OK : BL_ERR_TIMEOUT;
  uint32_t words[kMostStatusWords];
  if (n > 0 && cudaMemcpy(words, reinterpret_cast<const uint32_t*>(ws) + 1, n * sizeof(uint32_t), cudaMemcpyDeviceToHost) != cudaSuccess)
    return BL_ERR_CUDA;
  for (uint32_t i = 0; i < n; ++i)
    if (words[i] != 0) return BL_ERR_TIMEOUT;
  return BL_OK;
}

int64_t bitlinear_debug_decode_fallbacks(void* stream) {
  if (cudaStreamSynchronize((cudaStream_t)stream) != cudaSuccess) return -1;
  unsigned int n = 0;
  if (gemv_decode_take_fallbacks(&n) != cudaSuccess) return -1;
  return (int64_t)n;
}

int64_t bitlinear_debug_window_fallbacks(void* stream) {
  if (cudaStreamSynchronize((cudaStream_t)stream) != cudaSuccess) return -1;
  unsigned int n = 0;
  if (window_take_fallbacks(&n) != cudaSuccess) return -1;
  return (int64_t)n;
}

bl_status bitlinear_debug_wait_limit(int64_t polls, int meet_skew) {
  g_debug_wait_polls.store(polls < 0 ? -1 : (long long)polls, std::memory_order_relaxed);
  g_debug_meet_skew.store(meet_skew ? 1 : 0, std::memory_order_relaxed);
  return BL_OK;
}

}  // extern "C"
