/*
 * pq.h -- C ABI of the B200 (sm_100a) quantized linear layer: W8A8 and W4A8.
 *
 * The library implements the quantized linear operator of a decoder LLM as the
 * paper's "Unified low-bit inference framework" section states it: activations are
 * quantized per token to INT8, multiplied with INT8 (or packed INT4) weights in
 * integer arithmetic, and the INT32 result is dequantized to FP16.  The quantizer is
 * the paper's Eq. 1-2 with symmetric scaling (no zero point).
 *
 * Conventions for every call
 *   - All data pointers are DEVICE pointers owned by the caller, 16-byte aligned.
 *     The library allocates and frees no device memory.
 *   - `stream` is a cudaStream_t passed as void* (NULL = the legacy default stream).
 *     Calls are asynchronous and stream-ordered; none synchronizes the device.
 *   - The kernels are launched with programmatic stream serialization: a call may begin its
 *     set-up while the kernel before it in the stream drains, and waits for that kernel's
 *     completion before it reads activations, codes or token scales and before it writes.
 *     Packed weights and weight scales are treated as constants of the model and may be
 *     read ahead of that wait: they must be complete before the operation that directly
 *     precedes the GEMM call in the stream begins.  pq_pack_w8 / pq_pack_w4 guarantee this
 *     for GEMM calls that follow them; a caller that writes weight buffers by other means
 *     puts any stream operation (or a synchronization) between that write and the GEMM.
 *   - Matrices are dense row-major: X/Q/Y have one token per row, W has one output
 *     channel per row (K contiguous).
 *   - The return value is a pq_status.  Argument errors are detected before anything
 *     is launched.  Nothing aborts, throws or traps; non-finite inputs are memory
 *     safe with unspecified results.
 *   - Every wait inside a kernel is bounded; if one expires the kernel records
 *     PQ_ERR_TIMEOUT in a device status word, waits (bounded) for the copies and MMAs it has
 *     in flight, and returns; the outputs of that call are then unspecified.
 *     pq_device_status() reads that word.
 *   - The library keeps no per-call state on the host: calls may be made from several host
 *     threads and on several streams at once.  The only memory a call shares with other calls
 *     is what the caller passes in (see `workspace` below).
 *   - Requires compute capability 10.0; anything else returns PQ_ERR_ARCH (there is
 *     no fallback path).
 */
#ifndef PQ_H_
#define PQ_H_

#include <stddef.h>
#include <stdint.h>

#if defined(__GNUC__)
#define PQ_API __attribute__((visibility("default")))
#else
#define PQ_API
#endif

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  PQ_OK = 0,
  PQ_ERR_NULL = 1,    /* a required pointer is NULL */
  PQ_ERR_SHAPE = 2,   /* a size is non-positive or violates a divisibility rule */
  PQ_ERR_ALIGN = 3,   /* a pointer is not 16-byte aligned */
  PQ_ERR_ARCH = 4,    /* the current device is not compute capability 10.0 */
  PQ_ERR_CUDA = 5,    /* a CUDA runtime/driver call or a launch failed */
  PQ_ERR_TIMEOUT = 6, /* a bounded wait inside a kernel expired (device status word) */
  PQ_ERR_LIMIT = 7    /* a size exceeds a stated maximum of the entry point */
} pq_status;

/* Static string for a status code. */
PQ_API const char* pq_status_str(int status);

/* Name of the CUDA error (e.g. "cudaErrorIllegalAddress") behind the most recent PQ_ERR_CUDA returned
 * to the calling host thread; "" if there was none.  Static string; diagnostic only. */
PQ_API const char* pq_last_cuda_error(void);

/* Shape rules shared by the calls below (else PQ_ERR_SHAPE):
 *   M >= 1, N >= 8 with N % 8 == 0, K >= 16 with K % 16 == 0, K < 131072 (so that
 *   K * 128 * 128 fits INT32); W4 additionally needs group == 128 and K % 128 == 0. */

/*
 * Per-token symmetric INT8 activation quantization (Eq. 1-2 with n = 8; one scale
 * per token over the feature dimension).  For each row m:
 *   a = max_k |X[m,k]|,  s_tok[m] = a / 127.5 (= 2a/255),
 *   Q[m,k] = clamp(rne(X[m,k] * (127.5 / a)), -128, 127),
 * evaluated in IEEE binary32 with round-half-to-even; an all-zero row gives scale 0
 * and codes 0.
 *   x_f16 [M,K] FP16 in;  q [M,K] INT8 out;  s_tok [M] FP32 out.
 */
PQ_API int pq_quantize_act(const void* x_f16, int64_t M, int64_t K, int8_t* q, float* s_tok,
                    void* stream);

/*
 * Offline per-output-channel INT8 weight quantization (Eq. 2 with n = 8, one scale
 * per output channel) into the layout the W8A8 GEMM reads.
 *   s_ch[n] = max_k |W[n,k]| / 127.5,  code = clamp(rne(W[n,k] / s_ch[n]), -128, 127).
 *   w_f16 [N,K] FP16 in;  wq: pq_packed_w8_bytes(N,K) bytes out (opaque);
 *   s_ch [N] FP32 out.
 */
PQ_API int pq_pack_w8(const void* w_f16, int64_t N, int64_t K, void* wq, float* s_ch, void* stream);

/*
 * Offline group-wise INT4 weight quantization (Eq. 2 with n = 4, one scale per output
 * channel and group of `group` consecutive k) into the packed layout the W4A8 GEMM
 * reads (two codes per byte along K).
 *   s = fp16(max_{k in g} |W[n,k]| / 7.5),  code = clamp(rne(W[n,k] / float(s)), -8, 7).
 *   w_f16 [N,K] FP16 in;  wp: pq_packed_w4_bytes(N,K) bytes out (opaque);
 *   s_grp_f16 [K/group, N] FP16 out (the scales of one K-group are contiguous over n).
 */
PQ_API int pq_pack_w4(const void* w_f16, int64_t N, int64_t K, int32_t group, void* wp,
               void* s_grp_f16, void* stream);

/*
 * SmoothQuant variant (Eq. 3: Y = (X S^-1)(S W), S = diag(s), s_j = max|X_j|^alpha / max|W_j|^(1-alpha),
 * alpha = 0.5 as in the paper's experiments).  The column factors are computed once, offline, from
 * calibration activations; at run time they cost one extra [K] FP32 vector read per call.
 *
 *   pq_col_absmax:     out[k] = max_r |A[r,k]| for A FP16 [R,K] row-major (R >= 1, K as for the
 *                      quantizer); out: [K] FP32.  Run it on calibration activations and on W.
 *   pq_smooth_scales:  s[k] = sqrt(x_absmax[k]) / sqrt(w_absmax[k]),  s_inv[k] = 1 / s[k]  (each a
 *                      correctly rounded FP32 operation); a channel with a zero maximum gets 1.
 *   pq_quantize_act_smooth: pq_quantize_act of X S^-1 -- every element is multiplied by s_inv[k] in
 *                      FP32 (not rounded to FP16) BEFORE the token maximum is taken.
 *   pq_pack_w8_smooth / pq_pack_w4_smooth: pq_pack_w8 / pq_pack_w4 of S W (W is [N,K], so s[k]
 *                      multiplies along K), same outputs and layouts.
 * s, s_inv: [K] FP32 device vectors, 16-byte aligned.  The GEMM calls are unchanged: codes and scales
 * produced by the smooth variants go into pq_gemm_w8a8 / pq_gemm_w4a8 as they are.
 */
PQ_API int pq_col_absmax(const void* a_f16, int64_t R, int64_t K, float* out, void* stream);
PQ_API int pq_smooth_scales(const float* x_absmax, const float* w_absmax, int64_t K, float* s, float* s_inv,
                            void* stream);
/* The same for a migration strength alpha = alpha_quarters / 4 (0 ... 4, else PQ_ERR_SHAPE):
 * s[k] = x_absmax[k]^alpha / w_absmax[k]^(1 - alpha), the quarter powers taken as square roots
 * (x^(1/4) = sqrt(sqrt(x)), x^(3/4) = sqrt(x) * sqrt(sqrt(x))) so that every step is a correctly rounded FP32
 * operation; alpha_quarters = 2 is pq_smooth_scales.  Any other factor vector a caller computes itself goes
 * into the quantizer and pack calls just the same. */
PQ_API int pq_smooth_scales_alpha(const float* x_absmax, const float* w_absmax, int64_t K, int32_t alpha_quarters,
                                  float* s, float* s_inv, void* stream);
PQ_API int pq_quantize_act_smooth(const void* x_f16, const float* s_inv, int64_t M, int64_t K, int8_t* q,
                                  float* s_tok, void* stream);
PQ_API int pq_pack_w8_smooth(const void* w_f16, const float* s, int64_t N, int64_t K, void* wq, float* s_ch,
                             void* stream);
PQ_API int pq_pack_w4_smooth(const void* w_f16, const float* s, int64_t N, int64_t K, int32_t group, void* wp,
                             void* s_grp_f16, void* stream);

/*
 * Static (calibrated) activation scale: the paper's accuracy runs quantize with "calibrated scales"
 * fixed ahead of time instead of the token's own maximum.  One scale for the whole tensor:
 *   code = clamp(rne(X[m,k] * (1 / s)), -128, 127)   (FP32; values beyond the range saturate),
 *   s_tok[m] = s for every token, so that the GEMM calls are used unchanged.
 * scale: DEVICE pointer to one FP32 value (it may be produced by a preceding kernel); s <= 0 gives
 * codes 0 and token scales 0.  No maximum pass: the kernel reads X once and is launched like
 * pq_quantize_act.
 */
PQ_API int pq_quantize_act_static(const void* x_f16, const float* scale, int64_t M, int64_t K, int8_t* q,
                                  float* s_tok, void* stream);

/*
 * The same with one calibrated scale per feature channel (the per-channel granularity the paper's
 * "Preliminary" section names), given as reciprocals:
 *   code = clamp(rne(X[m,k] * inv_s[k]), -128, 127)   (one FP32 product; inv_s[k] <= 0 gives code 0),
 *   s_tok[m] = 1: a scale that depends on k cannot be taken out of the sum over k, so the caller folds
 *   s[k] = 1 / inv_s[k] into the weights (pq_pack_w8_smooth / pq_pack_w4_smooth with that vector, as for
 *   Eq. 3) and uses the GEMM calls unchanged.
 * inv_s: [K] FP32 device vector, 16-byte aligned.
 */
PQ_API int pq_quantize_act_static_channel(const void* x_f16, const float* inv_s, int64_t M, int64_t K, int8_t* q,
                                          float* s_tok, void* stream);

/*
 * The MLP's gated activation fused with the down projection's activation quantizer.  The paper
 * quantizes all linear layers of a decoder and reports whole prefill passes (its latency table), but
 * does not define the activation between the gate/up linears and the down linear; the gated form
 * SwiGLU is taken:  h[m,i] = silu(gate[m,i]) * up[m,i],  silu(g) = g / (1 + e^-g).
 * h is evaluated in FP32 as a FIXED sequence of single correctly rounded operations (the argument of
 * the exponential clamped to [-87, 88]; the reduction t = n ln2 + r, the degree-7 Taylor polynomial p
 * of e^r in Horner form with fused multiply-adds, d = fma(p, 2^n, 1) = 1 + e^t; then the IEEE reciprocal
 * of d, the product g * (1 / d) and one product with `up`), because its value decides integer codes;
 * it is not rounded to FP16.  Then pq_quantize_act's rule (Eq. 1-2 per token) is applied to h.
 * One pass: 4 bytes read and 1 written per element, instead of an FP16 round trip of h plus a
 * separate quantizer pass.
 *   gate_f16, up_f16 [M,I] FP16 in (the outputs of the gate and up linears);  q [M,I] INT8 out;
 *   s_tok [M] FP32 out;  I as K of the quantizer, I <= 16384 (PQ_ERR_SHAPE beyond).
 */
PQ_API int pq_swiglu_quantize(const void* gate_f16, const void* up_f16, int64_t M, int64_t I, int8_t* q,
                              float* s_tok, void* stream);

/*
 * Hadamard variant (Eq. 4: Y = (X H)(H^T W), H a normalized Hadamard matrix).  With W stored [N,K]
 * both operands are rotated along K: (X H)(W H)^T = X W^T.  Where K is a power of two (up to 16384) H
 * is the Sylvester matrix of order K itself.  For other layer widths (11008 = 2^8 * 43) no construction
 * is at hand, and H = I (x) H_B / sqrt(B) is block diagonal, H_B the Sylvester matrix of order
 * B = the largest power of two dividing K, at most 256.  pq_hadamard_block(K) returns the order used
 * (K or B).  The rotation is the in-place butterfly (distances 1, 2, ..., B/2 in this order) in FP32
 * on the exact FP16 inputs, times 1/sqrt(B); the rotated values are quantized from FP32.
 *   pq_quantize_act_hadamard: pq_quantize_act of X H (on line, fused into the quantizer kernel);
 *   pq_pack_w8_hadamard / pq_pack_w4_hadamard: pq_pack_w8 / pq_pack_w4 of W H (off line).
 * Same arguments, outputs and layouts as the plain calls; K <= 16384 (PQ_ERR_SHAPE beyond).  The
 * GEMM calls are unchanged.  pq_hadamard_block is a host-only query (0 for a K the quantizer rejects).
 */
PQ_API int32_t pq_hadamard_block(int64_t K);
PQ_API int pq_quantize_act_hadamard(const void* x_f16, int64_t M, int64_t K, int8_t* q, float* s_tok,
                                    void* stream);
PQ_API int pq_pack_w8_hadamard(const void* w_f16, int64_t N, int64_t K, void* wq, float* s_ch, void* stream);
PQ_API int pq_pack_w4_hadamard(const void* w_f16, int64_t N, int64_t K, int32_t group, void* wp,
                               void* s_grp_f16, void* stream);

PQ_API size_t pq_packed_w8_bytes(int64_t N, int64_t K);
PQ_API size_t pq_packed_w4_bytes(int64_t N, int64_t K);

/* Recover the integer codes from the opaque layouts as row-major INT8 [N,K]
 * (W4 codes lie in [-8,7]).  For checking and interchange; not on the hot path. */
PQ_API int pq_unpack_w8(const void* wq, int64_t N, int64_t K, int8_t* codes, void* stream);
PQ_API int pq_unpack_w4(const void* wp, int64_t N, int64_t K, int8_t* codes, void* stream);

/*
 * W8A8 linear ("weight layout, dequantization logic and matrix multiplication" of the
 * framework section; weight-activation quantization runs the product itself in
 * integers):
 *   ACC[m,n] = sum_k Q[m,k] * Wq[n,k]                      exact, INT32
 *   Y[m,n]   = fp16( float(ACC[m,n]) * s_tok[m] * s_ch[n] )
 *   q [M,K] INT8, s_tok [M] FP32 (from pq_quantize_act);  wq, s_ch [N] (from pq_pack_w8);
 *   y_f16 [M,N] FP16 out.
 * Any M is accepted; small M (decode shapes) is routed to a weight-streaming schedule
 * that computes the same result.
 *
 * workspace / workspace_bytes: optional scratch of THIS call (NULL / 0 = none).  With few output
 * tiles and a long K (e.g. a 7B-class layer at M = 512) the GEMM cuts K into parts that run on
 * different SMs; the parts' INT32 partial accumulators pass through the workspace and are summed
 * exactly, so the result does not depend on it.  Without a workspace, or with one too small for the
 * shape, K is simply not split.  (The paper's "matrix multiplication ... within the operator
 * template library" leaves scheduling to the kernel; this is scheduling only.)
 *   - Device memory owned by the caller, 256-byte aligned (else PQ_ERR_ALIGN), of at least
 *     pq_workspace_bytes(...) bytes for the shape to be served in full.
 *   - Before its first use it is prepared once with pq_workspace_init (which zeroes its first
 *     64 KB, the arrival counters); every call that completes leaves it prepared for the next.
 *     After a PQ_ERR_TIMEOUT prepare it again.
 *   - Calls that may overlap on the GPU (different streams, parallel graph branches) must be
 *     given different workspaces; calls ordered in one stream may share one.
 */
PQ_API int pq_gemm_w8a8(const int8_t* q, const float* s_tok, const void* wq, const float* s_ch,
                 int64_t M, int64_t N, int64_t K, void* y_f16, void* workspace, size_t workspace_bytes,
                 void* stream);

/*
 * The whole path of one linear in one call: per-token quantization of the FP16 activations (Eq. 1-2,
 * exactly pq_quantize_act) followed by pq_gemm_w8a8 / pq_gemm_w4a8 on the result.  Y is bit for bit what
 * the two calls give.  For the smallest decode shapes (one to four tokens, where the CUDA-core row
 * kernel is the schedule) the GEMM kernel quantizes its tokens itself and nothing else is launched: a
 * decode step is a chain of dependent launches, and each launch costs microseconds whatever it does.
 *   x_f16 [M,K] device; q_tmp int8 [M,K] and s_tok_tmp float [M]: device buffers of the caller for the
 *   codes and scales (written when two kernels run; their contents are unspecified afterwards);
 *   everything else as in pq_gemm_w8a8 / pq_gemm_w4a8.  On an argument error nothing is launched.
 */
PQ_API int pq_linear_w8a8(const void* x_f16, const void* wq, const float* s_ch, int64_t M, int64_t N,
                          int64_t K, void* y_f16, int8_t* q_tmp, float* s_tok_tmp, void* workspace,
                          size_t workspace_bytes, void* stream);
PQ_API int pq_linear_w4a8(const void* x_f16, const void* wp, const void* s_grp_f16, int32_t group,
                          int64_t M, int64_t N, int64_t K, void* y_f16, int8_t* q_tmp, float* s_tok_tmp,
                          void* stream);

/*
 * W4A8 linear: INT4 codes are widened to INT8 inside the kernel, multiplied in
 * integers per K-group and dequantized per group into an FP32 running sum:
 *   ACC_g[m,n] = sum_{k in group g} Q[m,k] * C[n,k]        exact, INT32
 *   R[m,n]     = sum_g float(ACC_g[m,n]) * float(s_grp[g,n])   (FP32, g ascending)
 *   Y[m,n]     = fp16( R[m,n] * s_tok[m] )
 *   wp, s_grp_f16 [K/group, N] from pq_pack_w4;  group must be 128.
 */
PQ_API int pq_gemm_w4a8(const int8_t* q, const float* s_tok, const void* wp, const void* s_grp_f16,
                 int32_t group, int64_t M, int64_t N, int64_t K, void* y_f16, void* stream);

/*
 * The exact INT32 accumulators of the two linears, computed by the same tensor-core
 * main loops as the calls above and written out instead of the FP16 result (for
 * parity checking).   acc [M,N];   acc_g [K/group, M, N] (group-major).
 */
PQ_API int pq_acc_w8a8(const int8_t* q, const void* wq, int64_t M, int64_t N, int64_t K, int32_t* acc,
                void* stream);
PQ_API int pq_acc_w4a8(const int8_t* q, const void* wp, int32_t group, int64_t M, int64_t N, int64_t K,
                int32_t* acc_g, void* stream);

/*
 * Several W8A8 linears over the SAME quantized tokens (the q/k/v projections, or gate and up, of
 * the layers the paper quantizes) as one call.  Result: exactly what `count` calls of pq_gemm_w8a8
 * with (wq[g], s_ch[g], N[g], y_f16[g]) give, bit for bit.  The members' output tiles are scheduled
 * together in a single kernel launch (of the weight-streaming kernel up to 128 tokens, and up to 256
 * where the members' 128-channel tiles x 2 token blocks do not exceed the number of SMs; of the
 * prefill kernel otherwise), which fills the SMs' waves across the members and pays the per-launch fixed cost
 * once -- at decode-shaped token counts that fixed cost is most of a call.
 *   count: 1..PQ_MAX_GROUP.  wq, s_ch, N, y_f16: HOST arrays of `count` entries (device pointers
 *   and column counts; read during the call, not retained).  q, s_tok, M, K as in pq_gemm_w8a8.
 *   The outputs must not overlap each other.  On an argument error nothing is launched.
 *   workspace / workspace_bytes: as for pq_gemm_w8a8 (sized with pq_workspace_bytes for the group).
 */
#define PQ_MAX_GROUP 4
PQ_API int pq_gemm_w8a8_group(const int8_t* q, const float* s_tok, int32_t count, const void* const* wq,
                              const float* const* s_ch, const int64_t* N, void* const* y_f16, int64_t M,
                              int64_t K, void* workspace, size_t workspace_bytes, void* stream);

/* The same for W4A8 linears (pq_gemm_w4a8 per member; one launch for all of them, except at M <= 128 when
 * the members together hold more 128-channel tiles than the device has SMs).  For M <= 128, and for M <= 256
 * when the members' 128-channel tiles x 2 token blocks do not exceed the number of SMs, the FP32
 * group sums of the K parts are added in a fixed order, but the number of parts depends on how many tiles
 * the launch holds, so the grouped result may differ from the per-member call in the last FP32 bit. */
PQ_API int pq_gemm_w4a8_group(const int8_t* q, const float* s_tok, int32_t count, const void* const* wp,
                              const void* const* s_grp_f16, int32_t group, const int64_t* N,
                              void* const* y_f16, int64_t M, int64_t K, void* stream);

/*
 * Workspace of the W8A8 calls (see pq_gemm_w8a8).
 *   pq_workspace_bytes: host-only (touches no device).  The number of bytes with which
 *     pq_gemm_w8a8 (count = 1) or pq_gemm_w8a8_group over the column counts N[0..count) at these M
 *     and K runs the schedule it would pick with unlimited room, on a GPU with `sms`
 *     multiprocessors (148 on a B200); 0 when that schedule does not split K (then no workspace is
 *     of any use) or when an argument is invalid.  The maximum over the shapes a caller issues
 *     serves all of them.  pq_gemm_w4a8 and every call that the weight-streaming kernel serves (M <= 128, narrow
 *     linears up to M = 256) need none.
 *   pq_workspace_init: zeroes the first 64 KB of `workspace` on `stream` (bytes >= 65536, 256-byte
 *     aligned).  GEMM calls enqueued afterwards on that stream (or after a synchronization) may
 *     use the workspace.  A buffer the caller has zero-filled by other means is equally good.
 */
PQ_API size_t pq_workspace_bytes(int64_t M, const int64_t* N, int32_t count, int64_t K, int32_t sms);
PQ_API int pq_workspace_init(void* workspace, size_t bytes, void* stream);

/*
 * Host-only query (touches no device): the schedule of the prefill kernel (the one pq_gemm_w8a8 uses
 * beyond the token counts of the weight-streaming kernel) on a GPU with
 * `sms` multiprocessors and a workspace of `scratch_bytes` (0 = none): the output tile
 * width (*tile_n = 256 or 128 columns) and the number of parts K is cut into (*k_parts, 1 = no
 * split).  For capacity planning and tests; the result has no effect on later calls.
 */
PQ_API int pq_plan_w8a8(int64_t M, int64_t N, int64_t K, int32_t sms, size_t scratch_bytes, int32_t* tile_n,
                        int32_t* k_parts);

/*
 * W8A8 linear for callers that cannot allocate device memory (the paper has no counterpart to
 * this call; it exists for deployment constraints, not for the method).
 *
 * Same result as pq_gemm_w8a8, same arguments without the workspace.  The difference is where the
 * split-K scratch comes from: not from a workspace argument -- which somebody had to cudaMalloc --
 * but from a fixed 32 MiB + 64 KiB array inside the library, held by every GPU that loads the
 * library until the process exits.  Meant for hosts that hand a plug-in nothing but its inputs and
 * outputs, for serving loops and capture regions in which cudaMalloc (a synchronizing call) is
 * off limits, and for programs that fix their whole device-memory budget at start-up.  The call
 * itself invokes no allocation or free routine of any kind.
 *   - Limit: M and N each rounded up to a multiple of 256, multiplied, may not exceed 2,097,152
 *     (e.g. 512 x 4096, 1024 x 2048, 256 x 8192); beyond that the call returns PQ_ERR_LIMIT and
 *     launches nothing.  M <= 128 needs no scratch: such calls are forwarded to pq_gemm_w8a8
 *     whatever N is, and the limit does not apply to them.
 *   - The first call on each device looks up the array's device address; make that first call
 *     outside any stream capture.
 *   - All calls on a device share the one array, and it keeps whatever the last call left in it
 *     (a call that completes restores the few words that must read zero; after a call that ended
 *     in PQ_ERR_TIMEOUT, pq_device_status() -- the call that reports it -- clears them with a memset
 *     on the array, so read the status before going on).  Two calls that overlap on the GPU
 *     -- different streams, parallel graph branches -- would race on it: keep them ordered.
 */
PQ_API int pq_gemm_w8a8_noalloc(const int8_t* q, const float* s_tok, const void* wq, const float* s_ch,
                                int64_t M, int64_t N, int64_t K, void* y_f16, void* stream);

/* ------------------------------------------------------------------------------------------------
 * Paged key/value cache and attention over it: what stands between the q/k/v linears of a decoder layer
 * and its output linear when many requests are served at once.  (The paper quantizes the linears and
 * times whole prefill and decode passes; it describes no cache.)
 *
 * A cache holds `pages` pages of `page` tokens for `heads` key/value heads of `dim` values:
 *   k, v              [pages, heads, page, dim]  FP16 (PQ_KV_F16) or INT8 codes (PQ_KV_INT8)
 *   k_scale, v_scale  [pages, heads, page]       FP32, PQ_KV_INT8 only (NULL otherwise): the scale of one
 *                                                token's vector of one head, value = code * scale;
 *                                                >= 0, as pq_kv_append writes it
 * A SLOT is page_id * page + offset.  Rules (else PQ_ERR_SHAPE): page a multiple of 16, at most 1024;
 * dim 64 or 128; 1 <= heads <= 1024; pages >= 1 and pages * heads * page < 2^31; type one of the two.
 */
#define PQ_KV_F16 0
#define PQ_KV_INT8 1
typedef struct {
  void* k;
  void* v;
  float* k_scale;
  float* v_scale;
  int64_t pages;
  int32_t heads;
  int32_t page;
  int32_t dim;
  int32_t type;
} pq_kv_cache;

/*
 * Block tables, slot map and positions of one step, built on the GPU from the requests' lengths.
 * Request b has kv_len[b] cached tokens and brings new_len[b] (either may be 0; a negative length counts
 * as 0).  With have = ceil(kv_len / page) and want = ceil((kv_len + new_len) / page), the want - have
 * pages it needs are taken from free_list in request order, beginning at *free_head:
 *   block_table [requests, width]  columns have .. want - 1 of every row are written, the others are left
 *   q_start [requests + 1]         exclusive prefix sums of new_len (row ranges of the step's tokens)
 *   kv_total [requests]            kv_len + new_len
 *   slots [tokens]                 where each new token's key and value go; -1 for rows beyond
 *                                  q_start[requests] and for tokens without a page
 *   pos [tokens]                   the token's position in its request; -1 beyond q_start[requests]
 *   free_next [1]                  *free_head + the pages needed (above free_count: the list was too short)
 * A token has no page when the free list is used up (its table entry becomes -1), when its column is
 * beyond `width`, or when the table's own entry is negative.  The caller gives `tokens` >= the sum of
 * new_len: tokens beyond are not mapped and pages that only they would begin are not entered.
 *   kv_len, new_len i32 [requests], free_list i32 [free_count], free_head i32 [1]: in.  free_next must not
 *   overlap free_head, nor kv_total kv_len (PQ_ERR_SHAPE when they are the same address).
 *   0 <= requests <= PQ_MAX_REQUESTS (PQ_ERR_LIMIT beyond), 0 <= tokens < 2^31, width >= 1, free_count >= 0.
 *   Index arrays need the alignment of their type only.
 */
#define PQ_MAX_REQUESTS 4096
PQ_API int pq_block_tables(const int32_t* kv_len, const int32_t* new_len, int64_t requests, int32_t* block_table,
                           int64_t width, const int32_t* free_list, int64_t free_count, const int32_t* free_head,
                           int32_t page, int64_t tokens, int32_t* q_start, int32_t* kv_total, int64_t* slots,
                           int32_t* pos, int32_t* free_next, void* stream);

/*
 * Writes the keys and values of `tokens` new tokens into the cache, token t at slots[t] (rows whose slot is
 * negative or beyond the cache are skipped; two rows with one slot leave a mixture of the two).  PQ_KV_INT8: every
 * (token, head) vector is quantized by the rule of pq_quantize_act (one scale over its `dim` values).
 *   k, v: FP16, row t at k + t * stride elements, heads * dim values each (stride >= heads * dim, a
 *   multiple of 8, so that slices of one wide q/k/v output serve as they are); 16-byte aligned.
 */
PQ_API int pq_kv_append(const pq_kv_cache* cache, const void* k_f16, int64_t k_stride, const void* v_f16,
                        int64_t v_stride, const int64_t* slots, int64_t tokens, void* stream);

/* The reverse: the values at `slots` as FP16 [tokens, heads, dim], dense (PQ_KV_INT8: code * scale in FP32,
 * rounded once; zeros where the slot is negative or beyond the cache).  For interchange and checking. */
PQ_API int pq_kv_read(const pq_kv_cache* cache, const int64_t* slots, int64_t tokens, void* k_f16, void* v_f16,
                      void* stream);

/*
 * Attention of the step's tokens over the paged cache, which already holds their own keys and values.
 * Row t of request b, q_start[b] <= t < q_start[b + 1], with n = q_start[b + 1] - q_start[b] rows and
 * L = kv_len[b] cached tokens, stands at position p = L - n + (t - q_start[b]) and sees the keys
 *   j <= p, j >= 0, and j > p - window when window > 0:
 *   s_j = scale * sum_d q[d] k_j[d],  y = sum_j e^(s_j - max) v_j / sum_j e^(s_j - max)
 * for query head h over the key/value head h / (heads / cache->heads).  Scores, maxima and sums are FP32, and so is
 * the sum of the products with the values.  For that product the weights (PQ_KV_INT8: times their value's scale) are
 * rounded to FP16, relative to the largest that the row sees: to 11 bits down to 2^-21 of it, below that to within
 * 2^-32 of it.  A row that sees no key (kv_len shorter than the chunk, window or not) gives 0.
 * A key that a row does not see does not reach it, whatever it holds, and nothing beyond kv_len or before
 * the window of a chunk's first row is used.  The VALUES in between are taken as finite: one that is infinite
 * or NaN also reaches rows of its request that do not see it (0 times it).
 *   q: FP16, row t at q + t * q_stride elements (a multiple of 8, >= heads * dim), heads * dim values
 *   block_table i32 [requests, width]; q_start i32 [requests + 1]; kv_len i32 [requests], tokens in the
 *     cache with the chunk's own (kv_total of pq_block_tables).  A page id outside the cache reads as
 *     zeros; keys beyond width * page are not seen.
 *   max_q, max_kv: bounds of the rows and the cached tokens of any request of this step, for the choice
 *     of the schedule.  A request with more rows than max_q leaves outputs unspecified; max_kv
 *     only steers how the keys are split.
 *   out: FP16 [tokens, heads, dim] dense.  Rows outside every request are left as they are.
 *   heads a multiple of cache->heads, heads / cache->heads <= 64; scale finite; window >= 0.
 *   workspace: as for pq_gemm_w8a8 (optional, prepared once with pq_workspace_init, one per stream of calls
 *     that may overlap): partial results of keys that are split over several SMs, summed in a fixed order.
 *     Without it, the keys of a request are not split; with too little, into fewer parts or not at all.
 * pq_attention_workspace_bytes: host-only; the workspace with which a call of these sizes without a window splits its
 *   keys as it would with unlimited room, for either type of cache; 0 when nothing is split or an argument is
 *   invalid.  pq_attention_workspace_bytes_window: the same with a window (0: none), which may want more or less.
 */
PQ_API int pq_paged_attention(const void* q_f16, int64_t q_stride, int32_t heads, const pq_kv_cache* cache,
                              const int32_t* block_table, int64_t width, const int32_t* q_start,
                              const int32_t* kv_len, int64_t requests, int64_t tokens, int64_t max_q,
                              int64_t max_kv, float scale, int32_t window, void* out_f16, void* workspace,
                              size_t workspace_bytes, void* stream);
PQ_API size_t pq_attention_workspace_bytes(int64_t requests, int64_t tokens, int64_t max_q, int64_t max_kv,
                                           int32_t heads, int32_t kv_heads, int32_t dim, int32_t sms);
PQ_API size_t pq_attention_workspace_bytes_window(int64_t requests, int64_t tokens, int64_t max_q, int64_t max_kv,
                                                  int32_t heads, int32_t kv_heads, int32_t dim, int32_t sms,
                                                  int32_t window);

/* ------------------------------------------------------------------------------------------------
 * Rotary positions.  The first `dim` values of every head of a row at position p are turned pair by pair; pair i,
 * 0 <= i < dim / 2, by p * freq[i] turns:
 *   (a, b) -> amplitude * (a cos - b sin, b cos + a sin)
 * with (a, b) the values i and i + dim / 2 (PQ_ROTARY_HALF) or 2 i and 2 i + 1 (PQ_ROTARY_PAIRS).  The values behind
 * the first `dim` are left as they are.  Angles are exact modulo a turn at every 32-bit position (negative ones turn
 * backwards); cosines, sines and products are FP32, and an FP16 result is rounded once.
 *   freq: DEVICE array [dim / 2], turns per position in units of 2^-64, 8-byte aligned; a constant of the model
 *   dim a multiple of 16, 16 .. 256; 2^-16 <= amplitude <= 2^16
 */
#define PQ_ROTARY_HALF 0
#define PQ_ROTARY_PAIRS 1
typedef struct {
  const uint64_t* freq;
  int32_t dim;
  int32_t layout;
  float amplitude;
} pq_rotary;

/*
 * Host-only (touches no device): the frequencies and the amplitude of a rotation.  Pair i makes base^(-2 i / dim)
 * radians per position, which `scaling` stretches by `factor` >= 1 for contexts beyond the `original` length:
 *   PQ_ROTARY_PLAIN   not at all
 *   PQ_ROTARY_LINEAR  all pairs by `factor`
 *   PQ_ROTARY_BASE    through the base: base * factor^(dim / (dim - 2))
 *   PQ_ROTARY_BANDS   pairs that make fewer than `low` turns over `original` positions by `factor`, those that make more
 *                     than `high` not, linearly in the pair's index in between; amplitude 0.1 ln(factor) + 1
 *   PQ_ROTARY_WAVES   the same by original / wavelength, linearly in it between `low` and `high`; amplitude 1
 * freq: HOST array [dim / 2], amplitude: one host float (1 but for BANDS).  Arguments that a scaling does not name are not
 * looked at; base > 1, 0 < low < high, original >= 1 (else PQ_ERR_SHAPE).
 */
#define PQ_ROTARY_PLAIN 0
#define PQ_ROTARY_LINEAR 1
#define PQ_ROTARY_BASE 2
#define PQ_ROTARY_BANDS 3
#define PQ_ROTARY_WAVES 4
PQ_API int pq_rotary_frequencies(int32_t dim, double base, int32_t scaling, double factor, double original, double low,
                                 double high, uint64_t* freq, float* amplitude);

/*
 * Rows of heads turned by their positions: head h of row t is `width` values at x + t * x_stride + h * x_head_stride and
 * goes to out + t * out_stride + h * out_head_stride (elements; FP16).
 *   width a multiple of 16, rotary->dim .. 1024; 1 <= heads <= 1024; strides multiples of 8, head strides >= width (with
 *   one head not looked at), out_stride >= width; 16-byte aligned.  out may be x with the same strides (in place), and may
 *   not overlap it otherwise.
 *   pos i32 [tokens]
 */
PQ_API int pq_rotate(const pq_rotary* rotary, const void* x_f16, int64_t x_stride, int64_t x_head_stride, int32_t heads,
                     int32_t width, const int32_t* pos, int64_t tokens, void* out_f16, int64_t out_stride,
                     int64_t out_head_stride, void* stream);

/*
 * pq_kv_append with the keys turned on the way, and the step's queries beside them, in one launch.  Keys are turned
 * over the first rotary->dim <= cache->dim values of a head; PQ_KV_INT8 quantizes the turned FP32 values.
 *   k, v, slots, tokens: as for pq_kv_append;  pos i32 [tokens]
 *   q: q_heads heads of cache->dim values per row, out: the same turned, both as for pq_rotate (q_heads 0: no queries, the
 *   pointers and strides are not looked at).  Queries are turned whatever their row's slot is.
 */
PQ_API int pq_kv_append_rotated(const pq_kv_cache* cache, const pq_rotary* rotary, const void* k_f16, int64_t k_stride,
                                const void* v_f16, int64_t v_stride, const int64_t* slots, const int32_t* pos,
                                int64_t tokens, const void* q_f16, int64_t q_stride, int64_t q_head_stride,
                                int32_t q_heads, void* out_f16, int64_t out_stride, int64_t out_head_stride, void* stream);

/* ------------------------------------------------------------------------------------------------
 * Latent attention: keys and values of all heads come from one latent vector a token, beside one rotary key of
 * PQ_LATENT_ROPE values that all heads share.  The cache holds a token's latent vector with its turned rotary key:
 *   data [pages, page, latent + PQ_LATENT_ROPE]  FP16
 * Slots and block tables are those of the paged key/value cache.  Rules (else PQ_ERR_SHAPE): latent 256 or 512; page a
 * multiple of 16, at most 1024; pages >= 1, pages * page < 2^31.
 */
#define PQ_LATENT_ROPE 64
typedef struct {
  void* data;
  int64_t pages;
  int32_t page;
  int32_t latent;
} pq_latent_cache;

/*
 * Writes the latent vectors and, turned by their positions, the rotary keys of `tokens` new tokens into the cache, token t
 * at slots[t] (rows whose slot is negative or beyond the cache are skipped; of two rows with one slot a mixture is
 * left), and turns the rotary part of the step's queries, in one launch.
 *   c: FP16, row t at c + t * c_stride (>= latent);  k_rope: FP16, row t at k_rope + t * k_rope_stride (>=
 *   PQ_LATENT_ROPE); strides multiples of 8, 16-byte aligned: slices of one linear's output serve as they are
 *   rotary->dim <= PQ_LATENT_ROPE;  slots i64, pos i32 [tokens]
 *   q, out: as for pq_kv_append_rotated, with heads of PQ_LATENT_ROPE values
 */
PQ_API int pq_latent_append(const pq_latent_cache* cache, const pq_rotary* rotary, const void* c_f16, int64_t c_stride,
                            const void* k_rope_f16, int64_t k_rope_stride, const int64_t* slots, const int32_t* pos,
                            int64_t tokens, const void* q_f16, int64_t q_stride, int64_t q_head_stride, int32_t q_heads,
                            void* out_f16, int64_t out_stride, int64_t out_head_stride, void* stream);

/* The reverse: latent vectors [tokens, latent] and turned rotary keys [tokens, PQ_LATENT_ROPE] at `slots`, dense (zeros
 * where a slot is negative or beyond the cache): what the expanded form multiplies out for tokens of earlier steps. */
PQ_API int pq_latent_read(const pq_latent_cache* cache, const int64_t* slots, int64_t tokens, void* c_f16, void* k_rope_f16,
                          void* stream);

/*
 * One matrix per head: y[t, h, :] = W[h] x[t, h, :], the products that take queries into the latent space (K values of a
 * head to N = latent) and results out of it (K = latent).  FP16 in and out, FP32 sums.
 *   x: head h of row t is K values at x + t * x_stride + h * x_head_stride;  w: dense [heads, N, K];
 *   y: N values at y + t * y_stride + h * y_head_stride
 *   K a multiple of 64 up to 512, N a multiple of 128 up to 1024, 1 <= heads <= 1024; strides as for pq_rotate, with K and
 *   N for the widths, and those of x below 2^38; y may not overlap x.  Unlike packed weights, w may be written by the operation right before the call.
 */
PQ_API int pq_head_linear(const void* x_f16, int64_t x_stride, int64_t x_head_stride, const void* w_f16, int32_t heads, int64_t N,
                          int64_t K, int64_t tokens, void* y_f16, int64_t y_stride, int64_t y_head_stride, void* stream);

/*
 * Latent attention, absorbed form: the step's queries in the latent space over the paged latent cache, which already holds
 * their own tokens.  Row t, head h of request b, with n = q_start[b + 1] - q_start[b] rows and L = kv_len[b] cached
 * tokens, stands at position p = L - n + (t - q_start[b]) and sees the tokens 0 <= j <= p:
 *   s_j = scale * q . data_j (latent + PQ_LATENT_ROPE values),  y = sum_j e^(s_j - max) data_j[: latent] / sum_j e^(s_j - max)
 * Precision, rows that see nothing (0), unusable page ids (zeros) and vectors that are not finite: as for
 * pq_paged_attention, the data taking the values' place.
 *   q: FP16 [tokens, heads, latent + PQ_LATENT_ROPE] dense;  out: FP16 [tokens, heads, latent] dense.  Rows outside every
 *     request are left as they are.  1 <= heads <= 1024, tokens * heads < 2^31; scale finite.
 *   block_table i32 [requests, width], q_start i32 [requests + 1], kv_len i32 [requests]: as for pq_paged_attention;
 *     width * page <= 2^30 and requests <= PQ_MAX_REQUESTS (else PQ_ERR_LIMIT)
 *   workspace: as for pq_gemm_w8a8; partial results of tokens that are split over several SMs, joined in a fixed order.
 *     The schedule is made on the GPU from the lengths.  Without a workspace, or with less than
 *     pq_latent_workspace_bytes, the tokens of a request are not split.
 * pq_latent_workspace_bytes: host-only; what every call of pq_latent_attention and pq_expanded_attention wants on a GPU
 *   with `sms` multiprocessors, whatever the sizes (0: sms < 1).
 */
PQ_API int pq_latent_attention(const void* q_f16, int32_t heads, const pq_latent_cache* cache, const int32_t* block_table,
                               int64_t width, const int32_t* q_start, const int32_t* kv_len, int64_t requests, int64_t tokens,
                               float scale, void* out_f16, void* workspace, size_t workspace_bytes, void* stream);
PQ_API size_t pq_latent_workspace_bytes(int32_t sms);

/*
 * Latent attention, expanded form: ragged queries over keys and values that have been multiplied out per head, as one
 * linear over the latent vectors gives them, beside the shared rotary key.  Row t of request b, with n = q_start[b + 1] -
 * q_start[b] rows and L = kv_start[b + 1] - kv_start[b] keys, stands at position p = L - n + (t - q_start[b]) and sees
 * the request's keys 0 <= j <= p; head h:
 *   s_j = scale * (q[: 128] . kv[j, h, : 128] + q[128 :] . k_rope[j]),  y = sum_j e^(s_j - max) kv[j, h, 128 :] / sum_j e^(s_j - max)
 * Precision, rows that see nothing (0) and values that are not finite: as for pq_paged_attention.
 *   q: FP16, row t at q + t * q_stride, heads * (128 + PQ_LATENT_ROPE) values (the rotary part last, turned)
 *   kv: FP16, row j at kv + j * kv_stride, heads * (128 + 128) values: a head's key, then its value
 *   k_rope: FP16, row j at k_rope + j * k_rope_stride, PQ_LATENT_ROPE values;  keys: rows of kv and k_rope
 *   strides multiples of 8, >= the row and below 2^38; 16-byte aligned;  requests <= PQ_MAX_REQUESTS (else PQ_ERR_LIMIT)
 *   q_start, kv_start i32 [requests + 1] within tokens and keys;  max_q: a bound of the rows of any request (a request
 *     with more leaves outputs unspecified)
 *   workspace: as for pq_latent_attention
 *   out: FP16 [tokens, heads, 128] dense.  Rows outside every request are left as they are.  1 <= heads <= 1024,
 *     tokens * heads < 2^31; scale finite.
 */
PQ_API int pq_expanded_attention(const void* q_f16, int64_t q_stride, int32_t heads, const void* kv_f16, int64_t kv_stride,
                                 const void* k_rope_f16, int64_t k_rope_stride, int64_t keys, const int32_t* q_start,
                                 const int32_t* kv_start, int64_t requests, int64_t tokens, int64_t max_q, float scale,
                                 void* out_f16, void* workspace, size_t workspace_bytes, void* stream);

/*
 * Reads the device status word of the current device into *host_status (PQ_OK or
 * PQ_ERR_TIMEOUT) and clears it.  Synchronizes the device; call it outside timed
 * regions.
 */
PQ_API int pq_device_status(int* host_status);

/*
 * The poll bound of the waits inside the kernels launched from now on (process-wide; 0 restores
 * the default of 2^24 polls, some 25 seconds: a poll of a barrier that nothing arrives on lasts 1.5
 * us, and a wait may have to outlast the kernel before in the stream).  For tests of the give-up path: with PQ_WAIT_NONE no
 * wait polls at all, so every role of a kernel gives up at its first wait although nothing is
 * wrong; with a bound of a few polls some wait runs out somewhere in the middle.  Either way the
 * kernel reports PQ_ERR_TIMEOUT through the status word and returns with unspecified outputs.
 */
#define PQ_WAIT_NONE 0xFFFFFFFFu
PQ_API int pq_set_wait_limit(uint32_t polls);

#ifdef __cplusplus
}
#endif
#endif /* PQ_H_ */
