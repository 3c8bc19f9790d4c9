/*
 * bitlinear.h - C ABI of the B200 (sm_100a) BitLinear forward library.
 *
 * BitLinear (BitNet, Sec. 2.1, Eq. 11):   y = W~ . Quant(LN(x)) . beta.gamma / Q_b
 *   step 1  LN(x) = (x - E x) / sqrt(Var x + eps)                         Eq. 12 (per group: Eq. 15)
 *   step 2  x~ = Clip(round(x^.Q_b/gamma), -(Q_b-1), Q_b-1), gamma = max|x^|   Eq. 4-5
 *           or Clip(round((x^-eta).Q_b/gamma), 0, Q_b-1), eta = min x^         Eq. 6
 *           (in this form gamma = max x^ - min x^, the range of the shifted values: a departure
 *           from Eq. 5 / 14 as printed, whose gamma = ||x||_inf would not map onto [0, Q_b];
 *           the gamma returned for BL_ETA is this range)
 *   step 3  W~ = Sign(W - alpha), alpha = mean W, beta = mean|W|          Eq. 1-3, 12 (per group: Eq. 13)
 *   step 4  acc = W~ x~ in exact integers, rescaled by beta.gamma/Q_b     Eq. 7, 11
 * Symbols follow the paper: M tokens, K input features (the contraction and the group
 * dimension), N output features, G groups along K (K_g = K/G), b = 8 bits, Q_b = 2^(b-1) = 128.
 *
 * Conventions that hold for every entry point unless it says otherwise
 *   - Every data pointer is a DEVICE pointer owned by the caller; matrices are dense row-major;
 *     base addresses are 16-byte aligned (BL_ERR_ALIGN otherwise).
 *   - The library allocates nothing and keeps no results between calls.  Scratch comes from the
 *     caller as (ws, ws_bytes); ask bitlinear_workspace_bytes() for the size.  The workspace
 *     may be reused by the next call on the same stream; it holds nothing the caller needs
 *     except the status word read by bitlinear_ws_status().  What the library does hold, per
 *     process: caches of device attributes and of per-kernel launch set-up (keyed by device
 *     ordinal), a call counter that makes the arrival tags of the cooperative LN+quant kernel
 *     unique, the setting of bitlinear_debug_wait_limit, and the fixed device array behind
 *     bitlinear_quant_act_noalloc.  None of it changes a result.
 *   - Calls are asynchronous on `stream` (a cudaStream_t passed as void*; NULL = default
 *     stream) and never synchronise.
 *   - Errors are detected on the host before any launch and returned as a bl_status; nothing
 *     is launched when the status is not BL_OK.  Kernels never trap or print.  A device-side
 *     wait that runs out of its iteration limit records BL_ERR_TIMEOUT in the workspace
 *     status word; outputs of that call are then undefined.
 *   - Rounding to integer codes and to 16-bit outputs is round-half-to-even.
 *   - Requirements on shapes: K % (8*G) == 0, 1 <= G <= BL_MAX_GROUPS, b == 8
 *     (Sec. 2.1 leaves other widths to future work: BL_ERR_UNSUPPORTED).
 */
#ifndef BITLINEAR_H_
#define BITLINEAR_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define BL_MAX_GROUPS 64

typedef enum {
  BL_OK = 0,
  BL_ERR_NULL = 1,        /* a required pointer is NULL */
  BL_ERR_SHAPE = 2,       /* a size is non-positive or breaks a divisibility rule */
  BL_ERR_ALIGN = 3,       /* a pointer is not 16-byte aligned */
  BL_ERR_UNSUPPORTED = 4, /* b != 8, unknown enum value, or layout not accepted by this call */
  BL_ERR_WORKSPACE = 5,   /* ws is NULL or smaller than bitlinear_workspace_bytes() */
  BL_ERR_CUDA = 6,        /* a CUDA runtime call (launch, attribute, tensor map) failed */
  BL_ERR_TIMEOUT = 7,     /* a bounded device-side wait expired (read via bitlinear_ws_status) */
  BL_ERR_TOO_LARGE = 8    /* the problem exceeds the built-in scratch of a *_noalloc entry point */
} bl_status;

typedef enum { BL_F32 = 0, BL_F16 = 1, BL_BF16 = 2, BL_I8 = 3 /* codes, where a call says so */ } bl_dtype;

/* Eq. 4-5 (signed codes in [-127,127]) or Eq. 6 (eta-shifted codes in [0,127]). */
typedef enum { BL_ABSMAX = 0, BL_ETA = 1 } bl_quant_mode;

/* Scope of gamma/eta (Sec. 2.1: per tensor in training, per token in inference).
 * PER_TENSOR: gamma, eta have G entries.  PER_TOKEN: M*G entries, index m*G + g. */
typedef enum { BL_PER_TENSOR = 0, BL_PER_TOKEN = 1 } bl_gran;

/* Storage order of the 1-bit weights W~ (bit = 1 means +1).
 *   CANONICAL  u8 [N, K/8]; weight k of row n is bit (k % 8) of byte n*K/8 + k/8.  Accepted by
 *              every entry point except gemv_decode; shapes are unrestricted.
 *   PREFILL    the same bits re-tiled for the tensor-core GEMM: blocks of 128 rows x 128
 *              weights, rows and K padded up to multiples of 128 (see bitlinear_packed_bytes and
 *              bitlinear_layout_index).  Needs K_g % 128 == 0.
 *   DECODE     the same bits re-ordered for the batch-1 GEMV.  Needs K % 256 == 0, N % 16 == 0. */
typedef enum { BL_LAYOUT_CANONICAL = 0, BL_LAYOUT_PREFILL = 1, BL_LAYOUT_DECODE = 2 } bl_layout;

typedef enum {
  BL_OP_BINARIZE_PACK = 0,
  BL_OP_QUANT_ACT = 1,
  BL_OP_FORWARD = 2,
  BL_OP_MATMUL_I32 = 3,
  BL_OP_MATMUL_DEQUANT = 4,
  BL_OP_BLOCK_FORWARD = 5,   /* M = batch * seq tokens, N = ffn width, K = model width d, G ignored (1) */
  BL_OP_FORWARD_LATENT = 6,
  BL_OP_GEMV_DECODE_BATCH = 7  /* bitlinear_gemv_decode_batch_ws; N and G ignored */
} bl_op;

/* Human-readable name of a status code (static string, never NULL). */
const char* bitlinear_status_string(bl_status st);

/* Bytes of scratch the given entry point needs for these sizes (0 on invalid sizes). */
size_t bitlinear_workspace_bytes(bl_op op, int64_t M, int64_t N, int64_t K, int G);

/* Bytes of the packed weight buffer for a layout (includes PREFILL padding); 0 if invalid. */
size_t bitlinear_packed_bytes(bl_layout layout, int64_t N, int64_t K);

/* Where weight (n, k) lives in a packed buffer of the given layout: writes the byte offset
 * and the bit number.  Host-only helper that documents the private layouts; tests use it to
 * map PREFILL/DECODE buffers back to CANONICAL.  Returns BL_ERR_SHAPE when out of range. */
bl_status bitlinear_layout_index(bl_layout layout, int64_t N, int64_t K, int64_t n, int64_t k,
                                 int64_t* byte_offset, int* bit);

/* Step 3, Eq. 1-3, 12, 13: alpha_g, beta_g over the K-slice g of all N rows, then
 * W~ = Sign(W - alpha_g) with Sign(0) = -1, packed 1 bit per weight.
 *   W         [N,K] of dtype wt (read twice).
 *   alpha_in  NULL, or G device floats used in place of the computed means (lets a caller
 *             fix alpha, e.g. to isolate the sign-and-pack step).
 *   W_packed  bitlinear_packed_bytes(layout,N,K) bytes, fully overwritten.
 *   alpha, beta  [G] fp32 outputs (the means in fp64, rounded once).
 *   rowsum    NULL or int32 [N,G]: sum over the group of W~[n,k] (used by eta_correction).
 * Sums are accumulated in fp64 in a fixed order, so results are run-to-run identical; the sign
 * test compares W against the fp64 mean exactly.  Workspace: BL_OP_BINARIZE_PACK. */
bl_status bitlinear_binarize_pack(const void* W, bl_dtype wt, int64_t N, int64_t K, int G,
                                  bl_layout layout, const float* alpha_in, uint8_t* W_packed,
                                  float* alpha, float* beta, int32_t* rowsum, void* ws,
                                  size_t ws_bytes, void* stream);

/* Steps 1-2, Eq. 12/15 then Eq. 4-6/14, b = 8.
 *   x      [M,K] of dtype xt.
 *   ln_eps LN epsilon; a negative value skips LN (codes are taken from x itself).
 *   x_q    int8 [M,K] codes.   gamma, eta: fp32, sized by gran (eta may be NULL for BL_ABSMAX).
 * gamma == 0 (constant input) yields all-zero codes, never NaN.  PER_TOKEN is one pass over x;
 * PER_TENSOR is two (statistics, then codes).  For segments of up to 8 KB that are a multiple of
 * 256 features both passes run in one cooperative kernel whose CTAs wait for one another between
 * the passes, with a limit: after a PER_TENSOR call bitlinear_ws_status(ws, stream) reports
 * BL_ERR_TIMEOUT if that wait expired (codes are then not written).  Workspace: BL_OP_QUANT_ACT.
 * PER_TOKEN needs no workspace (ws may be NULL).  Given one of at least 256 bytes, its first word
 * becomes the call's status word and segments of the shape above are fetched with bulk copies whose
 * bounded wait reports there (bitlinear_ws_status as above); the values written are the same. */
bl_status bitlinear_quant_act(const void* x, bl_dtype xt, int64_t M, int64_t K, int G, int b,
                              bl_quant_mode mode, bl_gran gran, float ln_eps, int8_t* x_q,
                              float* gamma, float* eta, void* ws, size_t ws_bytes, void* stream);

/* bitlinear_quant_act for callers that cannot provide a workspace.  (The paper has no counterpart:
 * this is a packaging variant of the entry point above, not another operation.)
 *
 * Who needs it: code that runs where device memory may not be allocated or sized at run time -
 * a plug-in called from inside another framework's stream callback or graph-building phase, a
 * real-time loop with a fixed memory budget, a host binding that only forwards pointers it was
 * given.  Such callers still own x, x_q, gamma and eta, but have nowhere to put the statistics
 * that the per-tensor path keeps between its two passes.
 *
 * The statistics go to a fixed array inside the library instead (24 bytes per segment for
 * BL_NOALLOC_MAX_SEGMENTS segments plus a 0.26 MB header, about 0.7 MB in all, resident on every
 * GPU that loads the library until the process ends).  Consequences:
 *   - BL_PER_TENSOR calls with M * G > BL_NOALLOC_MAX_SEGMENTS return BL_ERR_TOO_LARGE and launch
 *     nothing.  BL_PER_TOKEN calls keep no statistics there and have no such limit; they use the
 *     array's first word as their status word only.
 *   - All calls on one GPU share the array.  BL_PER_TENSOR calls that may overlap on the GPU
 *     (different streams) race on it and corrupt each other; keep them on one stream or order them
 *     yourself.  Overlapping BL_PER_TOKEN calls share nothing but the status word (each clears it
 *     when it starts), so their outputs are unaffected, but a timeout report of one may be wiped
 *     by the other.  A call leaves nothing behind that the next one depends on.
 *   - The first call on each device looks up the array's device address
 *     (cudaGetSymbolAddress); make that first call outside any stream capture.
 *   - No cudaMalloc, cudaFree or other allocating routine is called, now or later.
 * Arguments, results, host-side error codes and rounding are otherwise exactly those of
 * bitlinear_quant_act; the same kernels run, so the outputs are bit-identical.  The one difference
 * is where a device-side timeout is reported: the status word lives in the library's array, which
 * the caller cannot pass to bitlinear_ws_status; bitlinear_noalloc_status reads it instead. */
#define BL_NOALLOC_MAX_SEGMENTS 16384
bl_status bitlinear_quant_act_noalloc(const void* x, bl_dtype xt, int64_t M, int64_t K, int G, int b,
                                      bl_quant_mode mode, bl_gran gran, float ln_eps, int8_t* x_q,
                                      float* gamma, float* eta, void* stream);

/* Synchronises `stream`, then reads the status word that the last bitlinear_quant_act_noalloc call on
 * the current device left in the library's array (the counterpart of bitlinear_ws_status for that
 * entry point; the paper has no counterpart).  BL_OK, BL_ERR_TIMEOUT (a bounded device-side wait of
 * that call ran out: its codes were not written), or BL_ERR_CUDA.  Allocates nothing. */
bl_status bitlinear_noalloc_status(void* stream);

/* Steps 1, 2, 4, Eq. 11: y = (W~ x~) . beta_g gamma / Q_b summed over groups in ascending order.
 *   eta_correction != 0 (BL_ETA only) adds eta.beta_g.rowsum[n,g], which undoes the shift of
 *   Eq. 6 in the output; 0 is Eq. 11 as printed.
 *   W_packed  CANONICAL (any shape, plain CUDA-core kernel) or PREFILL (tcgen05 tensor-core
 *             kernel); beta [G] and rowsum [N,G] as produced by bitlinear_binarize_pack.
 *   y      [M,N] of dtype yt.
 * Workspace: BL_OP_FORWARD (holds the int8 codes, gamma, eta and the status word). */
bl_status bitlinear_forward(const void* x, bl_dtype xt, int64_t M, int64_t K, int64_t N, int G,
                            int b, bl_quant_mode mode, bl_gran gran, float ln_eps,
                            int eta_correction, const uint8_t* W_packed, bl_layout layout,
                            const float* beta, const int32_t* rowsum, void* y, bl_dtype yt,
                            void* ws, size_t ws_bytes, void* stream);

/* The layer as it runs in training (Sec. 2.2, "mixed precision training": the latent weights are
 * binarised on the fly during the forward pass): Eq. 1-3 on the high-precision W of this step,
 * then Eq. 11, in one call.  Nothing of the packed form outlives the call except what the caller
 * asks back.
 *   W [N,K] of dtype wt (the latent weights).  Other arguments as for bitlinear_forward.
 *   alpha_out, beta_out  NULL or fp32 [G]: the alpha_g and beta_g of this step (the straight-through
 *                        backward pass needs beta).
 * The packed weights live in the workspace, in PREFILL order when the shape allows the tensor-core
 * kernel (K % 128 == 0 per group), else CANONICAL.  y is bit-identical to bitlinear_binarize_pack
 * followed by bitlinear_forward.  Workspace: BL_OP_FORWARD_LATENT. */
bl_status bitlinear_forward_latent(const void* x, bl_dtype xt, const void* W, bl_dtype wt, int64_t M, int64_t K,
                                   int64_t N, int G, int b, bl_quant_mode mode, bl_gran gran, float ln_eps,
                                   int eta_correction, float* alpha_out, float* beta_out, void* y, bl_dtype yt,
                                   void* ws, size_t ws_bytes, void* stream);

/* Step 4 alone, Eq. 7: acc[g,m,n] = sum over k in group g of W~[n,k] . x_q[m,k], exact int32.
 * The parity hook for "accumulators are bit-exact when fed given codes".
 *   x_q [M,K] int8;  acc int32 [G,M,N].  Layout CANONICAL or PREFILL as for bitlinear_forward.
 * Workspace: BL_OP_MATMUL_I32. */
bl_status bitlinear_matmul_i32(const int8_t* x_q, int64_t M, int64_t K, int64_t N, int G,
                               const uint8_t* W_packed, bl_layout layout, int32_t* acc, void* ws,
                               size_t ws_bytes, void* stream);

/* Step 4 with the Eq. 11 rescale, for codes the caller already holds (the second half of
 * bitlinear_forward; lets one LN+Quant of x feed several weight matrices, e.g. Q, K and V).
 *   x_q [M,K] int8;  gamma, eta as written by bitlinear_quant_act for the same (mode, gran);
 *   eta may be NULL unless eta_correction != 0.  Other arguments as for bitlinear_forward.
 * The result is bit-identical to bitlinear_forward on the x that produced the codes.
 * Workspace: BL_OP_MATMUL_DEQUANT. */
bl_status bitlinear_matmul_dequant(const int8_t* x_q, int64_t M, int64_t K, int64_t N, int G,
                                   bl_gran gran, const float* gamma, const float* eta,
                                   int eta_correction, const uint8_t* W_packed, bl_layout layout,
                                   const float* beta, const int32_t* rowsum, void* y, bl_dtype yt,
                                   void* ws, size_t ws_bytes, void* stream);

/* bitlinear_matmul_dequant with output-side options, for fusing what follows a BitLinear in the
 * decoder block (Sec. 2, Fig. 2b) into its epilogue, and for weights whose alpha / beta are taken
 * per block of output features (the partitioning of Sec. 2.1 "Model parallelism with Group
 * Quantization", Eq. 13, applied along N: each device's slice of output features carries its own
 * alpha and beta; also how W_q, W_k, W_v stacked into one [3d, d] matrix keep their own beta).
 *   beta_rows  output features per beta block: beta is [N / beta_rows, G] (block-major), rowsum
 *              stays [N, G].  0 means one block (beta [G]).  Must divide N and be a multiple of 32.
 *   relu       non-zero: y = max(y, 0), applied before the residual.
 *   residual   NULL or [M, N] of dtype yt with row stride ld_res (elements): y += residual.
 *              May alias y only if ld_res == ld_y and residual == y (each element is read by
 *              the thread that then writes it).
 *   ld_y       row stride of y in elements (0 means N), so y may be a column block of a wider buffer.
 * With epi == NULL or all-zero options the call equals bitlinear_matmul_dequant. */
typedef struct {
  int64_t beta_rows;
  int relu;
  const void* residual;
  int64_t ld_res;
  int64_t ld_y;
} bl_epilogue;
bl_status bitlinear_matmul_dequant_ex(const int8_t* x_q, int64_t M, int64_t K, int64_t N, int G,
                                      bl_gran gran, const float* gamma, const float* eta,
                                      int eta_correction, const uint8_t* W_packed, bl_layout layout,
                                      const float* beta, const int32_t* rowsum, const bl_epilogue* epi,
                                      void* y, bl_dtype yt, void* ws, size_t ws_bytes, void* stream);

/* bitlinear_binarize_pack for NB blocks of N / NB consecutive output features, each with its own
 * alpha_g and beta_g (Eq. 13 applied along N, see bitlinear_matmul_dequant_ex): block j is
 * binarised against the mean of its own rows.
 *   alpha, beta  [NB, G];  alpha_in NULL or [NB, G];  rowsum NULL or [N, G].
 *   W_packed     the blocks' packed images one after the other, which for PREFILL (N / NB a
 *                multiple of 128) and CANONICAL / DECODE layouts is the packed image of the
 *                whole [N, K] matrix.
 * Runs one pass of bitlinear_binarize_pack per block on `stream`; the workspace is that of one
 * block (BL_OP_BINARIZE_PACK), reused in stream order. */
bl_status bitlinear_binarize_pack_nsplit(const void* W, bl_dtype wt, int64_t N, int64_t K, int G, int NB,
                                         bl_layout layout, const float* alpha_in, uint8_t* W_packed,
                                         float* alpha, float* beta, int32_t* rowsum, void* ws,
                                         size_t ws_bytes, void* stream);

/* Steps 1, 2, 4 for one token (M = 1), fused in a single kernel that streams the packed
 * weights once; Eq. 11 with per-token gamma.  W_packed must be in DECODE layout.
 *   x [K] of dtype xt;  y [N] of dtype yt.  K % 256 == 0, K <= 32768, N % 16 == 0, and for G > 1
 *   K_g % 128 == 0 (BL_ERR_SHAPE otherwise).  No workspace.
 * The weights are constants of the model and are read AHEAD of stream order: the kernel starts
 * copying W_packed into shared memory while earlier work on `stream` may still be running
 * (programmatic dependent launch), so whatever wrote W_packed must have completed before this
 * call is made (a pack on the same stream: synchronise once after packing).  x, beta, rowsum
 * and y are only touched in stream order.
 * The one device-side wait (for those copies) is bounded; if it ever ran out, the affected warps
 * read their weights from global memory instead, so there is no status to collect and y is the
 * same either way. */
bl_status bitlinear_gemv_decode(const void* x, bl_dtype xt, int64_t K, int64_t N, int G, int b,
                                bl_quant_mode mode, float ln_eps, int eta_correction,
                                const uint8_t* W_packed, const float* beta,
                                const int32_t* rowsum, void* y, bl_dtype yt, void* stream);

/* bitlinear_gemv_decode for a small batch: M tokens (decode with a few sequences in flight, the
 * per-token inference of Sec. 2.1 with one weight stream shared by the batch).  Each token gets
 * its own LN statistics, gamma and eta (Eq. 12, 4-6 per token); up to 8 tokens share one pass
 * over the packed weights (tensor-core mma on bit planes of the packed words), larger M runs
 * ceil(M/8) passes with the weights served from L2.  For M >= 2 a token's result does not depend on
 * what else is in the batch (same bits); M == 1 is handed to the kernel of bitlinear_gemv_decode,
 * which is faster for one token and may differ from this one in the last bit of gamma.  W_packed
 * is read ahead of stream order, as there.
 *   x [M,K] of dtype xt;  y [M,N] of dtype yt;  W_packed in DECODE layout.
 *   K % 256 == 0, (K/G) % 256 == 0, N % 16 == 0, min(M, 8) * (K + 16) <= 155 KB (BL_ERR_SHAPE otherwise).
 * No workspace; no device-side waits for M >= 2. */
bl_status bitlinear_gemv_decode_batch(const void* x, bl_dtype xt, int64_t M, int64_t K, int64_t N, int G,
                                      int b, bl_quant_mode mode, float ln_eps, int eta_correction,
                                      const uint8_t* W_packed, const float* beta, const int32_t* rowsum,
                                      void* y, bl_dtype yt, void* stream);

/* bitlinear_gemv_decode_batch with a workspace (Sec. 2.1, Eq. 12, 4-7, 11 per token), for G == 1,
 * eta_correction == 0, M >= 2 and K <= 12288: two kernels per call.  The first quantises the tokens
 * once (one CTA per token; LN statistics, gamma / eta, codes: the fp32 arithmetic of the kernel of
 * bitlinear_gemv_decode) into the workspace.  The second streams the packed weights once and
 * multiplies: for up to 8 tokens the bit-plane kernel of bitlinear_gemv_decode_batch, told to take
 * codes, gamma and code sums from the workspace instead of quantising every token in every CTA; for
 * more, the tcgen05 tensor cores (weight bit planes written to tensor memory as the A operand, int32
 * accumulators, exact), one pass per 32 tokens (per 16 when K > 6144), so that the time of a call
 * depends little on M up to 32.  A token's result does not depend on what else is in the batch, nor
 * on which of the two product kernels ran (same bits).  Other shapes, G > 1 and eta_correction are
 * handed to bitlinear_gemv_decode_batch's own path where it takes the shape (of the workspace only
 * the status word is used: cleared; its shape rules apply); M == 1 to the kernel of
 * bitlinear_gemv_decode, whose sums run in another order (same codes up to the tolerated ties,
 * gamma to the last bit or so).
 *   x [M,K] of dtype xt;  y [M,N] of dtype yt;  W_packed in DECODE layout, read ahead of stream
 *   order as there.  K % 256 == 0, N % 16 == 0.
 * Workspace: BL_OP_GEMV_DECODE_BATCH (device memory, 16-byte aligned; its first word is the status
 * word of bitlinear_ws_status: the tensor-core kernel's waits are bounded, and BL_ERR_TIMEOUT there
 * means y of this call is not valid).  The workspace holds the codes between the two kernels, so
 * calls that may overlap (different streams) need workspaces of their own. */
bl_status bitlinear_gemv_decode_batch_ws(const void* x, bl_dtype xt, int64_t M, int64_t K, int64_t N, int G,
                                         int b, bl_quant_mode mode, float ln_eps, int eta_correction,
                                         const uint8_t* W_packed, const float* beta, const int32_t* rowsum,
                                         void* y, bl_dtype yt, void* ws, size_t ws_bytes, void* stream);

/* Causal self-attention core of the decoder block (Sec. 2, Fig. 2b; the paper keeps it in high
 * precision): per batch and head O = softmax(Q K^T / sqrt(d_h) + causal mask) V, fp16 in and out,
 * fp32 softmax statistics and accumulators.  No positional encoding.
 *   q, k, v  fp16 [batch*seq, heads*128] with a common row stride ld (elements), so they may be
 *            column blocks of one buffer;  o fp16, same shape, row stride ld_o.
 *   head_dim must be 128, seq a multiple of 64, ld and ld_o multiples of 8. */
bl_status bitlinear_attention_causal(const void* q, const void* k, const void* v, void* o, int batch, int seq,
                                     int heads, int head_dim, int64_t ld, int64_t ld_o, void* stream);

/* One BitNet decoder block, forward (Sec. 2, Fig. 2b): every linear map is a BitLinear (its own
 * LN + per-token 8-bit quantisation in front, Eq. 11), the attention core and the residual adds
 * stay in fp16:
 *     q, k, v = BitLinear_{Q,K,V}(x)            (one LN + quant of x feeds all three)
 *     a       = causal attention(q, k, v)
 *     h       = x + BitLinear_O(a)
 *     u       = ReLU(BitLinear_up(h))
 *     y       = h + BitLinear_down(u)           (down uses the eta form of Eq. 6 on its input)
 * d = heads * 128; FFN width ffn; tokens T = batch * seq (seq % 64 == 0); d % 128 == 0, ffn % 128 == 0.
 * All weight buffers are PREFILL-packed with one group: W_q, W_k, W_v, W_o [d,d], W_up [ffn,d],
 * W_down [d,ffn]; beta_* point to one float each (as written by bitlinear_binarize_pack).
 * Every intermediate is a caller buffer (fp16, row-major), so each stage can be inspected:
 *   q, k, v [T,d] with row stride ld_qkv (0 means d);  a, h [T,d];  u [T,ffn];  y [T,d].
 * ReLU and the two residual adds run in the epilogues of the up, O and down GEMMs.  Q, K and V run
 * as ONE GEMM over a [3d, d] weight matrix when the caller lays them out for it: W_k directly
 * behind W_q and W_v behind W_k in memory (likewise beta_q, beta_k, beta_v, as written by
 * bitlinear_binarize_pack_nsplit with NB = 3), and q, k, v the three column blocks of one
 * [T, 3d] buffer (k = q + d, v = q + 2d, ld_qkv = 3d); otherwise as three GEMMs.  The values
 * written are the same either way.  9 launches in the fused layout, 11 otherwise.
 * Workspace: BL_OP_BLOCK_FORWARD (codes, gamma, eta, quant and GEMM scratch).  Asynchronous on
 * `stream`; bitlinear_ws_status(ws, stream) reports a device-side timeout of any of the block's
 * kernels (the first one clears the status word, the later ones only ever set it). */
typedef struct {
  const uint8_t *W_q, *W_k, *W_v, *W_o, *W_up, *W_down;
  const float *beta_q, *beta_k, *beta_v, *beta_o, *beta_up, *beta_down;
} bl_block_weights;
typedef struct {
  void *q, *k, *v, *a, *h, *u;
  int64_t ld_qkv;
} bl_block_buffers;
bl_status bitlinear_block_forward(const void* x, int batch, int seq, int heads, int64_t ffn, float ln_eps,
                                  const bl_block_weights* w, const bl_block_buffers* buf, void* y, void* ws,
                                  size_t ws_bytes, void* stream);

/* ---- attention at inference: positions, windows, a key/value cache held in 4 bits --------------
 * What a BitNet decoder needs around its BitLinear layers to answer token by token (Sec. 2, Fig. 2b
 * keeps this part in high precision; Sec. 2.1 leaves its form open).  Token rows are [T, heads *
 * head_dim] with a row stride in elements, so inputs may be column blocks of one fused buffer; query
 * head h reads key/value head h / (heads / kv_heads).  Types are BL_F16 and BL_BF16 unless said
 * otherwise (BL_ERR_UNSUPPORTED), row strides multiples of 8.  Indices that live in device memory
 * (positions, slots, page numbers, lengths) cannot be checked on the host: what each kernel does with
 * one out of range is stated, and no access leaves the buffers described by the arguments. */

/* Norm of each query and key head with the position rotation, in one pass:
 *   x^ = w . x / sqrt(mean(x^2) + eps)   over the head's head_dim values (eps < 0: no norm, no weight; not NaN)
 *   (x^_a, x^_b) -> (x^_a cos t - x^_b sin t, x^_b cos t + x^_a sin t),   t = position . inv_freq[i]
 * for the pairs i < rot_dim / 2: a = i, b = i + rot_dim / 2, or a = 2i, b = 2i + 1 when interleaved
 * != 0; values from rot_dim on are only normalised.  fp32 throughout, angles reduced in fp64 (so far
 * positions lose nothing), one rounding at the end.
 *   q [T, heads * head_dim] stride ld_q, k [T, kv_heads * head_dim] stride ld_k, dtype dt (also BL_F32).
 *   head_dim a multiple of 16, 16..256; rot_dim a multiple of 16, 0..head_dim.
 *   wq, wk      [head_dim] of dtype dt, or NULL (ones).
 *   inv_freq    fp32 [rot_dim / 2];  positions int32 [T]: a negative one marks a row of padding, whose
 *               outputs are left as they were.
 *   q_out, k_out  strides ld_qo, ld_ko; may be q, k themselves (same strides), else must not overlap them.
 * T = 0 is valid and does nothing.  No workspace. */
bl_status bitlinear_qk_norm_rope(const void* q, const void* k, bl_dtype dt, int64_t T, int heads, int kv_heads,
                                 int head_dim, int64_t ld_q, int64_t ld_k, const void* wq, const void* wk,
                                 float eps, int rot_dim, int interleaved, const float* inv_freq,
                                 const int32_t* positions, void* q_out, void* k_out, int64_t ld_qo, int64_t ld_ko,
                                 void* stream);

/* Attention of prompts with a sliding window and sinks (first tokens that stay visible):
 *   o_i = sum_j p_ij v_j,   p_i = softmax over the visible j of scale . q_i . k_j
 * where position i sees j <= i with i - j < window or j < sinks (window <= 0: every j <= i).
 *   batch sequences.  cu_q, cu_k: int32 [batch + 1] first rows of the sequences in q / o and in k / v
 *   (packed prompts of different lengths), or NULL: sequence b owns rows b * seq_q .. (seq_k for keys).
 *   cu_k may be NULL with cu_q given: the key rows are then those of cu_q.  seq_q, seq_k: the common
 *   length, or with cu_* an upper bound of the lengths (rows of a sequence beyond it are not
 *   processed).  rows_q, rows_k: rows present in q / o and k / v; entries of cu_* are clamped to them, and
 *   must not decrease (else which rows are processed is not defined).
 *   A sequence with fewer query rows than key rows has its queries at the last positions (a chunk
 *   behind tokens that are already known); with more, the first ones see nothing.  A query that sees
 *   nothing gets zeros; one whose visible scores have no softmax (a NaN or +infinity among them, or nothing
 *   but -infinity) NaN.  Rows of o outside every sequence are left as they were.
 *   head_dim 64 or 128; heads a multiple of kv_heads; scale 0..2e38, 0 means 1 / sqrt(head_dim).
 * Values in invisible places have no influence, whatever they are (infinities and NaN included).
 * fp32 softmax statistics and accumulators; probabilities are rounded to the type of v for the
 * product, and one rounding on output.  The kernel's waits are bounded; if one ever ran out, the rows concerned are
 * computed another way (same result up to rounding), so there is no status to collect.
 * o must not overlap q, k or v.  batch = 0 or seq_q = 0 is valid and does nothing.  No workspace. */
bl_status bitlinear_attention_window(const void* q, const void* k, const void* v, void* o, bl_dtype dt, int batch,
                                     const int32_t* cu_q, const int32_t* cu_k, int64_t seq_q, int64_t seq_k,
                                     int64_t rows_q, int64_t rows_k, int heads, int kv_heads, int head_dim,
                                     int64_t ld_q, int64_t ld_k, int64_t ld_v, int64_t ld_o, int window, int sinks,
                                     float scale, void* stream);

/* A paged key/value cache held in 4 bits: Eq. 6 with 4-bit codes, per token and head.
 *   eta = min x,  step = (max x - min x) / 15  (both rounded to dtype),  code = clip(round((x - eta) /
 *   step), 0, 15),  value = eta + step . code.  step == 0 stores code 0.  A row that holds a non-finite
 *   value is stored as NaN (step and eta) as a whole.
 * pages: num_pages x bitlinear_kv4_page_bytes() bytes; a page holds page_size tokens (16, 32 or 64) of all
 * heads.  Within a page, head h owns page_size * (head_dim + 8) contiguous bytes:
 *   key codes    [page_size][head_dim / 2]: byte j of a token holds values 2j (low nibble) and 2j + 1
 *   value codes  [page_size / 8][8][4][head_dim / 32][2][2]: octet of tokens, eighth of the row, pair of
 *                tokens, word, token of the pair, bytes: value d of token t sits in octet t / 8, eighth
 *                d / (head_dim / 8), pair t % 8 / 2, word d % (head_dim / 8) / 4, token t % 2, nibble d % 4
 *   key (step, eta) [page_size][2] of dtype, then value (step, eta) likewise.
 * (The attention kernel's operands come out of these orders with one mask per pair of values.)
 * A slot is page * page_size + place in the page. */
typedef struct {
  void* pages;
  int64_t num_pages;
  int page_size, kv_heads, head_dim;   /* head_dim 64 or 128 */
  bl_dtype dtype;                      /* BL_F16 or BL_BF16: type of step and eta, and of the rows in and out */
} bl_kv4_cache;

/* Bytes of one page (0 if a size is not supported). */
size_t bitlinear_kv4_page_bytes(int page_size, int kv_heads, int head_dim);

/* Quantises T tokens' key and value rows (stride ld_k, ld_v, dtype of the cache) into the cache at
 * slots int64 [T]; a slot outside the cache (e.g. -1: padding) is skipped.  No slot may appear twice in
 * a call.  The codes are those of exact arithmetic on the rounded step and eta.  T = 0 does nothing. */
bl_status bitlinear_kv4_append(const bl_kv4_cache* cache, const void* k, const void* v, int64_t T, int64_t ld_k,
                               int64_t ld_v, const int64_t* slots, void* stream);

/* The values the cache holds at slots int64 [T] (in any order, repeats allowed), rounded to its dtype;
 * rows of k, v whose slot is outside the cache are left as they were.  T = 0 does nothing. */
bl_status bitlinear_kv4_read(const bl_kv4_cache* cache, void* k, void* v, int64_t T, int64_t ld_k, int64_t ld_v,
                             const int64_t* slots, void* stream);

/* Attention of the last n_q tokens of each sequence over the cache (one token per step, or a few
 * drafted ones being checked), with the visibility rule of bitlinear_attention_window.
 *   q, o [batch * n_q, heads * head_dim] of the cache's dtype, strides ld_q, ld_o.
 *   block_table int32 [batch, max_pages]: page of each run of page_size tokens.  Entries whose tokens
 *   no query sees are not read; tokens of an entry outside 0..num_pages-1 are invisible.
 *   lens int32 [batch]: tokens of the sequence in the cache, the n_q new ones included (clamped to
 *   0..max_pages * page_size).  Query i of n_q stands at position lens - n_q + i; one that sees nothing
 *   (negative position, empty sequence) gets zeros.
 *   A query whose visible scores have no softmax (a NaN or +infinity among them, or nothing but -infinity) gets NaN.
 *   scale as there.  n_q >= 1, any number; made for few.
 * Sums and statistics in fp32.  Rounded for the products: the query to fp16 after a power of two per row (exact
 * but for values 2^-24 of the row's largest and less), probability times value step to fp16 (after a power of
 * two); one rounding on output.  The work is split along the sequences over the whole GPU and joined in a
 * fixed order (same inputs and sizes, same bits).  o must not overlap q or the cache.  batch = 0 does nothing.
 * Workspace: bitlinear_attention_kv4_ws_bytes() (16-byte aligned; bitlinear_ws_status reads its start: the
 * kernel's waits for its copies are bounded, and BL_ERR_TIMEOUT there means that one ran out; the rows of o
 * that miss tokens for it are NaN); calls that may overlap need workspaces of their own. */
bl_status bitlinear_attention_kv4(const void* q, int batch, int n_q, int heads, int64_t ld_q, const bl_kv4_cache* cache,
                                  const int32_t* block_table, int64_t max_pages, const int32_t* lens, int window,
                                  int sinks, float scale, void* o, int64_t ld_o, void* ws, size_t ws_bytes,
                                  void* stream);
size_t bitlinear_attention_kv4_ws_bytes(int batch, int n_q, int heads, int kv_heads, int head_dim);   /* 0 if a size is not supported */

/* Copies whole pages inside the cache, in every layer: for each pair (src, dst) of pairs int32 [n][2],
 * page dst becomes a copy of page src (a forked sequence's last page, a copy on write, the moves of a
 * compaction).  Layer l's pages start at pages + l * layer_stride bytes.  A pair with a page outside
 * 0..num_pages-1 is skipped.  No page may be the destination of two pairs, nor the destination of one
 * and the source of another (the order of the copies is not defined).  page_bytes and layer_stride
 * are multiples of 16, layer_stride >= num_pages * page_bytes (any value for one layer).  n = 0 does nothing. */
bl_status bitlinear_kv4_copy_pages(void* pages, size_t page_bytes, int64_t num_pages, int layers, size_t layer_stride,
                                   const int32_t* pairs, int64_t n, void* stream);

/* ---- layers held in 8 bits, and experts made of them -------------------------------------------
 * The layers of a BitNet that are not binarised (Sec. 2 keeps its other components "high-precision, e.g.
 * 8-bit": the output layer first of all), and a feed-forward block of experts of which each token visits a few.
 *   matrix of codes  int8 [rows, K], a scale (fp32) per row: value = scale . code, code in -127..127
 *   tokens' rows come from bitlinear_rms_norm_quant; a weight matrix [N, K] is one too, a scale per output channel,
 *   and bitlinear_rms_norm_quant with eps < 0 quantises it.
 * Indices in device memory (rows, offsets, places) cannot be checked on the host: what each kernel does with
 * one out of range is stated, and no access leaves the buffers described by the arguments.  Rows of a token that are
 * not finite stay visible as NaN. */

/* Residual's addition, root-mean-square norm, 8-bit codes with a scale per token, in one pass:
 *   h_t = residual_t + x_t,  or with rows:  h_t = residual_t + sum_j row_weights[t, j] . x[rows[t, j]]   (j < top_k)
 *   y_t = weight . h_t / sqrt(mean(h_t^2) + eps)         (eps < 0: y = h, no norm, no weight; not NaN)
 *   scale_t = max |y_t| / 127,   code = round(y_t / scale_t)       (half to even)
 *   x [x_rows, K] stride ld_x, dtype dt (BL_F32, BL_F16, BL_BF16; residual, weight, h, y likewise).  Without rows x_rows >= T.
 *   rows int32 [T, top_k] (an entry outside 0..x_rows-1, e.g. -1, adds nothing), row_weights fp32 [T, top_k] or NULL (ones);
 *   top_k 1..64, the places and weights of bitlinear_route_topk serve: x is then what the experts left.
 *   residual [T, K] stride ld_res, or NULL.  weight [K] or NULL (ones).
 *   h, y [T, K] strides ld_h, ld_y, x_q int8 [T, K] stride ld_q with scale fp32 [T]: each may be NULL if not wanted,
 *   but not all.  h and y may be residual, or without rows x, themselves (same stride), else outputs overlap nothing.
 *   K a multiple of 8, 8..32768; strides multiples of 8.
 * fp32 throughout, also for rows whose squares or products with the weights leave its range (they are scaled by powers of
 * two for it); the codes are those of h before it is rounded to dt, and those of exact arithmetic where y / scale is
 * further than 2^-13 from a border between two codes (with rows: and further than the roundings of the sum of
 * top_k + 1 terms).  A row of zeros has codes and scale 0; a row in which a value is not finite has scale NaN and codes 0.
 * T = 0 does nothing.  No workspace. */
bl_status bitlinear_rms_norm_quant(const void* x, bl_dtype dt, int64_t x_rows, int64_t T, int64_t K, int64_t ld_x,
                                   const int32_t* rows, const float* row_weights, int top_k, const void* residual,
                                   int64_t ld_res, const void* weight, float eps, void* h, int64_t ld_h, void* y,
                                   int64_t ld_y, int8_t* x_q, int64_t ld_q, float* scale, void* stream);

/* Matrix product of codes with a scale per token and per output channel:
 *   y[m, n] = (sum_k x_q[m, k] w_q[n, k]) . x_scale[m] . w_scale[n] + bias[n],  ReLU,  + residual[m, n]
 *   x_q int8 [M, K] stride ld_x, w_q int8 [N, K] stride ld_w: K a multiple of 16, 16..131056, strides multiples of 16
 *   (codes may be -128..127: no sum leaves 32 bits).  x_scale fp32 [M], w_scale fp32 [N], either NULL: ones.
 *   bias [N] or NULL, residual [M, N] stride ld_res or NULL, y [M, N] stride ld_y, all of dtype yt (BL_F32, BL_F16,
 *   BL_BF16), element-aligned.  y may be residual itself (same stride), else overlaps nothing.  N 1..2^24.
 * All inputs are read in the stream's order: w_q may be written just before the call by any kernel on the same stream.
 * The sums are exact; then fp32, one rounding on output.  A NaN stays one through the ReLU.  Waits are bounded; were one
 * to run out, the rows concerned are NaN.  M = 0 does nothing.  No workspace. */
bl_status bitlinear_matmul_i8(const int8_t* x_q, int64_t M, int64_t K, int64_t N, int64_t ld_x, const float* x_scale,
                              const int8_t* w_q, int64_t ld_w, const float* w_scale, const void* bias, int relu,
                              const void* residual, int64_t ld_res, void* y, bl_dtype yt, int64_t ld_y, void* stream);

/* The experts of each token, and the lists of rows that they make.
 *   logits [T, experts] stride ld, dtype dt (BL_F32, BL_F16, BL_BF16), element-aligned; experts 1..512.
 *   chosen   int32 [T, top_k]: the experts with the top_k largest scores, largest first; of equal scores the lowest index
 *            (-0 and 0 are equal, a NaN counts as less than -infinity).  top_k 1..32, at most experts.
 *   weights  fp32 [T, top_k]: exp(z - max z) of the chosen over its sum over the chosen (normalise != 0) or over all
 *            experts.  Where that is no number (a NaN anywhere, +infinity, nothing but -infinity): NaN.
 *   offsets  int32 [experts + 1]: rows offsets[e] .. offsets[e + 1] - 1 of the list belong to expert e.
 *   rows     int32 [T * top_k]: the token of each row of the list, ordered by expert, then by token.
 *   places   int32 [T, top_k]: the row of the list that belongs to each choice.
 *   positions int32 [T] or NULL: a negative one marks a row of padding (as in bitlinear_qk_norm_rope), which visits no expert:
 *            chosen and places -1, weights 0; entries of rows behind offsets[experts] are then left as they were.
 * T = 0 sets offsets to 0.  T * top_k <= 2^30.  Workspace: bitlinear_route_topk_ws_bytes() (0 for up to 64 tokens: ws may
 * be NULL), 16-byte aligned; calls that may overlap need workspaces of their own. */
bl_status bitlinear_route_topk(const void* logits, bl_dtype dt, int64_t T, int experts, int64_t ld, int top_k,
                               int normalise, const int32_t* positions, int32_t* chosen, float* weights,
                               int32_t* offsets, int32_t* rows, int32_t* places, void* ws, size_t ws_bytes,
                               void* stream);
size_t bitlinear_route_topk_ws_bytes(int64_t T, int experts);      /* 0 if a size is not supported, too */

/* Matrix products of lists of rows, each with the weights of its expert:
 *   y[r, n] = (sum_k x[rows[r], k] w[e, n, k]) . x_scale[rows[r]] . w_scale[e, n] + bias[e, n],  ReLU
 * for the rows r of expert e, offsets[e] <= r < offsets[e + 1].  Lists may be empty or hold every row.
 *   x [x_rows, K] stride ld_x, w [experts, N, K] with row stride ld_w and expert_stride a
 *   multiple of it (at least N ld_w; any for one expert), both of type `operand`:
 *     BL_I8    codes; x_scale fp32 [x_rows], w_scale fp32 [experts, N], either NULL: ones.  K as in bitlinear_matmul_i8.
 *     BL_F16, BL_BF16   values (x_scale and w_scale NULL): fp32 sums.  K a multiple of 8, 8..2^20, strides multiples of 8.
 *   offsets int32 [experts + 1], experts 1..1024: clamped to 0..R; one below an offset before it counts as that one.
 *   rows int32 [R] (clamped to 0..x_rows-1), or NULL: row r of x itself, x_rows >= R.
 *   bias [experts, N] or NULL, y [R, N] stride ld_y, of dtype yt (BL_F32, BL_F16, BL_BF16), element-aligned; y overlaps nothing.
 *   N 1..2^24.  Rows of y outside every list are left as they were.
 * fp32 sums are formed in an order that the sizes alone decide (same inputs, same bits).  One rounding on output; NaN and
 * waits as in bitlinear_matmul_i8.  R = 0 does nothing.  No workspace. */
bl_status bitlinear_matmul_grouped(const void* x, bl_dtype operand, int64_t x_rows, int64_t K, int64_t N, int64_t ld_x,
                                   const float* x_scale, const void* w, int64_t ld_w, int64_t expert_stride,
                                   const float* w_scale, int experts, const int32_t* offsets, const int32_t* rows,
                                   int64_t R, const void* bias, int relu, void* y, bl_dtype yt, int64_t ld_y,
                                   void* stream);

/* Synchronises `stream`, then reads the status that a previous bitlinear_forward,
 * bitlinear_matmul_i32 or other call that names it left at the start of `ws` (a word, or words
 * of which any may report).  BL_OK, BL_ERR_TIMEOUT, or BL_ERR_CUDA. */
bl_status bitlinear_ws_status(const void* ws, void* stream);

/* Test and diagnostic hook: caps the number of polls that the bounded device-side waits of
 * kernels launched afterwards by this process may make (bitlinear_gemv_decode's wait for its
 * weight copies; the waits of bitlinear_attention_window, bitlinear_attention_kv4, bitlinear_matmul_i8 and
 * bitlinear_matmul_grouped; the meeting between the
 * two passes of the cooperative per-tensor kernel of bitlinear_quant_act).  polls < 0 restores the built-in limits; 0 means a single poll (for
 * bitlinear_gemv_decode and bitlinear_attention_window: none at all, weights are read from global
 * memory, rows are computed one by one; for bitlinear_attention_kv4: none, it reports the timeout and its rows
 * are NaN; for the two matrix products: none, their rows are NaN).
 * meet_skew != 0 additionally makes the cooperative kernel wait for an arrival tag that no CTA
 * publishes, so that its wait runs out by construction: the kernel then records
 * BL_ERR_TIMEOUT in the status word, writes no codes and returns (nothing hangs, traps or
 * faults).  Process-wide and not synchronised with calls in flight on other host threads; not for
 * production use.  Always returns BL_OK. */
bl_status bitlinear_debug_wait_limit(int64_t polls, int meet_skew);

/* Test and diagnostic hook: synchronises `stream`, then returns and clears the number of warps of
 * bitlinear_gemv_decode kernels (on the current device, since the last call of this function) whose
 * bounded wait for a stage of weights ran out, so that they read the stage from global memory
 * instead.  The result of such a call is still correct, only slow; a healthy run returns 0.
 * -1 on a CUDA error. */
int64_t bitlinear_debug_decode_fallbacks(void* stream);

/* The same for bitlinear_attention_window: the number of CTAs whose bounded waits ran out, so that they
 * computed their rows over the visible places one by one. */
int64_t bitlinear_debug_window_fallbacks(void* stream);

#ifdef __cplusplus
}
#endif
#endif /* BITLINEAR_H_ */
