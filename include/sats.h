/*
 * sats.h -- C ABI of the GB300 (sm_103a) library for the runtime path of
 * "Sensitivity-Aware Thresholding and Token Routing for Activation
 * Sparsification in Large Language Models" (arXiv 2607.08991).
 *
 * The path: the CATS-thresholded gated MLP (Sec. 2, Eqs. 1-5; SATS, Sec. 3.1,
 * keeps this runtime mask and only chooses the per-layer threshold t_l), run
 * under per-token routing between the base (dense) and sparse MLP through a
 * vocabulary lookup table (Sec. 3.2, Eq. 13 and Fig. 2), chained over a
 * stack of decoder MLP blocks with RMSNorm and a residual add.
 *
 * Conventions for every call
 *   - Matrices follow the paper's row-vector convention y = x W: W_gate and
 *     W_up are [H][N] (hidden x intermediate), W_down is [N][H]; activations
 *     are [B][H].  All arrays are row-major and contiguous.
 *   - bf16 data is passed as its 16-bit patterns (const void*, 2 bytes each).
 *   - Pointers marked "device" are CUDA device pointers on the current device;
 *     "host" pointers are ordinary host memory.  The caller owns every buffer
 *     it passes; the library keeps no pointer to caller memory after a call
 *     returns, except that work it enqueued on `stream` reads/writes them.
 *   - `stream` is a cudaStream_t (NULL = legacy default stream).  Every call
 *     that takes a stream only enqueues work on it and returns without
 *     synchronising, unless stated otherwise.
 *   - Argument errors are detected on the host and returned before anything is
 *     enqueued.  Errors found by a kernel (a token id outside the vocabulary, a
 *     wait that ran out of time) are recorded in a status word in the
 *     workspace (or in the caller's status word for sats_route) and returned by
 *     sats_get_error; a call that synchronises returns them itself.
 *     sats_gate_act and sats_gate_act_f32 have no status word: a wait that
 *     runs out leaves NaN in a.  No call aborts, throws, or traps on the device.
 *   - Calls never allocate device memory, except sats_layer_create,
 *     sats_lora_create and sats_q4_create.
 *   - Requirements: H a multiple of 8 and 8 <= H <= 8192; N >= 1; B >= 0.
 *   - SM occupancy: the single-token / two-token decode kernel (the small-batch
 *     path of sats_sparse_mlp and the calls built on it) runs one CTA on every
 *     SM (about 216 KB of shared memory each) and its CTAs wait, bounded, for
 *     one another's prologue.  It needs every SM to become free while it runs:
 *     a kernel on another stream that holds SMs for longer than 2 s (a
 *     persistent kernel, or one spinning on a flag) makes the call give up with
 *     SATS_ETIMEOUT from sats_get_error, and y and the index lists are then
 *     incomplete.  Ordinary kernels on other streams only delay the call.  The
 *     kernel is not launched cooperatively: that guarantees co-residency but
 *     stops the next call from starting on SMs this call frees, which measured
 *     8 us slower per call on the Llama-shaped layer.
 */
#ifndef SATS_H
#define SATS_H

#include <stddef.h>
#include <stdint.h>

#if defined(__GNUC__)
#define SATS_API __attribute__((visibility("default")))
#else
#define SATS_API
#endif

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    SATS_OK = 0,
    SATS_EINVAL = 1,    /* null pointer, negative size, NaN or negative threshold, bad k */
    SATS_ESHAPE = 2,    /* H not a multiple of 8, H or N out of range */
    SATS_ECUDA = 3,     /* a CUDA runtime call failed (launch, copy, allocation) */
    SATS_EDEVICE = 4,   /* a kernel reported bad input (token id outside [0, V)) or an internal fault */
    SATS_ETIMEOUT = 5,  /* a bounded device-side wait gave up */
    SATS_ENOSPACE = 6   /* workspace smaller than sats_workspace_bytes() */
} sats_status;

/* Opaque handle of one MLP block; owns its repacked device weights. */
typedef struct sats_layer sats_layer;
typedef struct sats_lora sats_lora;
typedef struct sats_q4 sats_q4;

/* Library version, (major << 16) | minor. */
SATS_API int sats_version(void);

/* Human-readable name of a status code (static string, never NULL). */
SATS_API const char *sats_status_string(sats_status s);

/*
 * sats_layer_create -- repack one gated-MLP block (Sec. 2, Eq. 1) for the
 * runtime path.
 *   W_gate, W_up : device bf16 [H][N];  W_down : device bf16 [N][H].
 * The handle stores two device arrays that it allocates (the only allocation
 * in this library): Wg_t [N][H] (row j = column j of W_gate) and
 * W_ud [N][2H] (row j = column j of W_up followed by row j of W_down), so that
 * the weights a kept neuron needs are one contiguous 4H-byte row and a
 * skipped neuron costs no memory traffic.  The repacking runs on `stream`;
 * the call synchronises `stream` before returning, after which the caller may
 * free the three source arrays.  *out receives the handle.
 */
SATS_API sats_status sats_layer_create(const void *W_gate, const void *W_up, const void *W_down,
                              int H, int N, void *stream, sats_layer **out);

/* Frees the handle's device arrays (synchronises the device first). */
SATS_API sats_status sats_layer_destroy(sats_layer *layer);

/* Reads back H and N of a layer (host outputs, may be NULL). */
SATS_API sats_status sats_layer_shape(const sats_layer *layer, int *H, int *N);

/*
 * Workspace.  Every compute call takes a device workspace `ws` of at least
 * sats_workspace_bytes(H, N, B) bytes (B = the largest batch the caller will
 * pass).  It holds scheduling counters, the device status word, the LoRA
 * path's partial sums (16 KB), one 64-bit word per 8 neurons (kept counts and
 * prefixes for the index outputs) and the routing scratch of sats_mlp_stack:
 * N bytes plus B * 5 plus about 19 KB.  A batch that runs on the
 * tensor cores (sats_uses_tensor_cores) also needs, per token, bf16 copies of
 * its activations and of h (two parts each) plus one keep byte per neuron:
 * about B * (4 H + 5 N) bytes more.  It must be
 * zero-filled once before first use (sats_workspace_init does that on
 * `stream`); every call leaves its counters at zero for the next call.  Calls
 * that share one workspace must not overlap on the GPU.
 */
SATS_API size_t sats_workspace_bytes(int H, int N, int B);
SATS_API sats_status sats_workspace_init(void *ws, size_t ws_bytes, void *stream);

/*
 * sats_sparse_mlp -- the CATS-thresholded gated MLP (Sec. 2, Eqs. 1-5):
 *   a = SiLU(x W_gate);  keep_j = |a_j| >= t_l;  y = ((keep * a) * (x W_up)) W_down
 * for each of B tokens, bf16 weights with fp32 accumulation.
 *
 * Two execution paths, chosen by batch size (sats_uses_tensor_cores):
 *  - small batches (B <= 2 for H <= 4096, B = 1 above) stream W_gate once per
 *    call and read only the W_up columns and W_down rows of kept neurons;
 *  - larger batches run as two tensor-core GEMMs over all neurons,
 *    [x W_gate | x W_up] and then h W_down, with the mask applied to
 *    h = CATS(SiLU(x W_gate)) * (x W_up) between them; h, and fp32
 *    activations, are carried as a bf16 high part plus a bf16 low part
 *    (about 16 significant bits) with fp32 accumulation.
 *   x          : device bf16 [B][H]
 *   t_l        : threshold, >= 0 (0 keeps every neuron: the dense MLP;
 *                +inf keeps none and gives y = 0).  NaN or < 0 -> SATS_EINVAL.
 *   y          : device fp32 [B][H], written.
 *   active_idx : device int32 [B][N] or NULL.  Row b receives the kept neuron
 *                indices of token b in increasing order (entries past the
 *                count are unspecified).
 *   active_cnt : device int32 [B] or NULL; the number of kept neurons per token.
 * active_idx and active_cnt must both be NULL or both be given.
 */
SATS_API sats_status sats_sparse_mlp(const sats_layer *layer, const void *x, int B, float t_l,
                            float *y, int32_t *active_idx, int32_t *active_cnt,
                            void *ws, size_t ws_bytes, void *stream);

/*
 * sats_sparse_mlp_fixed_scratch -- sats_sparse_mlp with no workspace argument,
 * for callers that cannot allocate device memory.  The paper has no
 * counterpart to this call.  Such callers include plug-ins whose host
 * application owns every device allocation through its own allocator, code
 * that runs where cudaMalloc is not permitted or would stall (it synchronises
 * the device), and plain C callers that link only this library and have no
 * device allocator at all.
 *
 * Arguments, results and errors are those of sats_sparse_mlp.  Instead of a
 * workspace the call uses one 256 KiB array in the library's device memory;
 * every GPU that loads the library holds this array until the process exits.
 * A call whose workspace would exceed the array, i.e. with
 * sats_workspace_bytes(H, N, B) > 256 KiB, is rejected with SATS_ENOSPACE
 * before anything is enqueued.  On the fused small-batch kernel (B <= 2 for
 * H <= 4096, B = 1 above) the workspace is one 64-bit word per 8 neurons plus
 * about 17 KB, which admits N up to about 245,000; a batch on the tensor-core
 * path (sats_uses_tensor_cores) also needs its staging (activations, h and
 * keep bytes per token, and padding to whole tiles), so only small layers fit
 * there: for example N <= 5504 at H = 8192, B = 2, and N <= 1008 at H = 4096,
 * B = 8.  The call allocates nothing: before its kernels it clears the
 * array's control words with cudaMemsetAsync on `stream`.
 *
 *   dev_status : device int32 [1] or NULL.  If given, it receives this call's
 *                device status word after the kernels, in stream order (0 when
 *                every bounded device wait completed); sats_get_status_word
 *                reads it back and returns SATS_OK, SATS_ETIMEOUT or
 *                SATS_EDEVICE.  Without it, device-side errors of this call (a
 *                bounded wait that gave up, leaving y and the index lists
 *                incomplete) are not reported.
 *
 * Each call looks up the array's device address on the current device
 * (cudaGetSymbolAddress, which neither allocates nor synchronises), so the
 * address is always that of the current device and context.  All calls share
 * the one array, so calls that can overlap on the GPU (on different streams,
 * or from several host threads without ordering) race and must be serialised
 * by the caller.
 */
SATS_API sats_status sats_sparse_mlp_fixed_scratch(const sats_layer *layer, const void *x, int B, float t_l,
                                                   float *y, int32_t *active_idx, int32_t *active_cnt,
                                                   int32_t *dev_status, void *stream);

/*
 * sats_uses_tensor_cores -- 1 if a call with batch B on a layer of hidden size
 * H runs on the tensor-core path described under sats_sparse_mlp (also for
 * sats_dense_mlp and for each block of sats_mlp_stack), 0 if it runs on the
 * fused small-batch kernel.  Pure host function.
 */
SATS_API int sats_uses_tensor_cores(int H, int B);

/*
 * sats_last_cuda_error -- text of the CUDA error behind the most recent
 * SATS_ECUDA returned on the calling host thread, with the step that failed
 * (a static or thread-local string, valid until the thread's next call).
 */
SATS_API const char *sats_last_cuda_error(void);

/* As sats_sparse_mlp, with fp32 activations x: device fp32 [B][H]. */
SATS_API sats_status sats_sparse_mlp_f32(const sats_layer *layer, const float *x, int B, float t_l,
                                float *y, int32_t *active_idx, int32_t *active_cnt,
                                void *ws, size_t ws_bytes, void *stream);

/*
 * sats_sparse_mlp_union, sats_sparse_mlp_union_f32 -- sats_sparse_mlp for a
 * batch of 3 to 8 tokens (H <= 4096), computed over the union of the tokens'
 * kept neurons: the gate runs over all neurons on the tensor cores; then only
 * neurons some token keeps have their W_up column and W_down row read, once for
 * the whole batch (Sec. 2, Eqs. 1-5 per token: each token still keeps exactly
 * its own neurons, so the result equals sats_sparse_mlp's).  This reads
 * 2HN (1 + 2 |U| / N) bytes instead of 6HN, |U| the union size, which pays
 * when the tokens' kept sets overlap strongly; for independent kept sets at
 * these batch sizes the default path of sats_sparse_mlp is faster.
 * Arguments, results and errors are those of sats_sparse_mlp (x bf16) and
 * sats_sparse_mlp_f32 (x fp32, carried as bf16 high and low parts), with a
 * workspace of sats_workspace_bytes(H, N, B); B outside [3, 8] or H > 4096
 * returns SATS_ESHAPE.
 */
SATS_API sats_status sats_sparse_mlp_union(const sats_layer *layer, const void *x, int B, float t_l, float *y,
                                           int32_t *active_idx, int32_t *active_cnt, void *ws, size_t ws_bytes,
                                           void *stream);
SATS_API sats_status sats_sparse_mlp_union_f32(const sats_layer *layer, const float *x, int B, float t_l,
                                               float *y, int32_t *active_idx, int32_t *active_cnt, void *ws,
                                               size_t ws_bytes, void *stream);

/*
 * LoRA-aware sparse path (Sec. 4, fine-tuned models: the sparse path of a routed
 * fine-tuned model runs the thresholded MLP on its adapted weights, with the
 * low-rank updates folded into the sparse kernel).  An adapter of rank r holds,
 * for each projection W of the block, factors A, B with W' = W + scale A B:
 *   A_gate, A_up [H][r], B_gate, B_up [r][N], A_down [N][r], B_down [r][H]
 * (device bf16, row-major; the adapter keeps its own packed copies, so the
 * caller may free them after sats_lora_create returns).  r is 8, 16, 24 or 32
 * (else SATS_ESHAPE); scale finite (else SATS_EINVAL).
 *
 * sats_sparse_mlp_lora computes, for each of B tokens,
 *   g = x W_gate + scale (x A_gate) B_gate,  a = SiLU(g),  keep = |a| >= t_l
 *   u = x W_up + scale (x A_up) B_up,        h = keep ? a u : 0
 *   y = h W_down + scale (h A_down) B_down
 * in the decode kernel: the gate's low-rank term for every neuron, the up and
 * down terms only for kept neurons.  Batches of 3 to 65535 tokens that
 * sats_uses_tensor_cores puts there, from hidden size 96, run on the tensor
 * cores in that kernel's fp32 accuracy and stream the weights once per 32
 * tokens: fp32 activations and h enter as three bf16 parts, and sums are
 * rounded to fp32 every 32 products (every 64 with fp32 activations in tiles
 * of more than 16 tokens).  Other batches run as passes of the decode kernel.
 * On the tensor cores a dropped neuron's W_down row is multiplied by zero
 * rather than not read, so it has to be finite there, as in sats_sparse_mlp's
 * batches.
 * Arguments, index outputs, workspace and errors are those of sats_sparse_mlp
 * (x bf16) and sats_sparse_mlp_f32 (x fp32); the adapter must match the
 * layer's H and N (else SATS_ESHAPE).
 */
SATS_API sats_status sats_lora_create(const sats_layer *layer, const void *A_gate, const void *B_gate,
                                      const void *A_up, const void *B_up, const void *A_down, const void *B_down,
                                      int r, float scale, void *stream, sats_lora **out);
SATS_API sats_status sats_lora_destroy(sats_lora *lora);
SATS_API sats_status sats_sparse_mlp_lora(const sats_layer *layer, const sats_lora *lora, const void *x, int B,
                                          float t_l, float *y, int32_t *active_idx, int32_t *active_cnt, void *ws,
                                          size_t ws_bytes, void *stream);
SATS_API sats_status sats_sparse_mlp_lora_f32(const sats_layer *layer, const sats_lora *lora, const float *x, int B,
                                              float t_l, float *y, int32_t *active_idx, int32_t *active_cnt,
                                              void *ws, size_t ws_bytes, void *stream);

/*
 * sats_dense_mlp -- the base gated MLP of Sec. 2, Eq. 1 (every neuron kept):
 *   x : device bf16 [B][H];  y : device fp32 [B][H].
 */
SATS_API sats_status sats_dense_mlp(const sats_layer *layer, const void *x, int B, float *y,
                           void *ws, size_t ws_bytes, void *stream);

/*
 * sats_route -- token routing by lookup table (Sec. 3.2, Eq. 13; Fig. 2).
 *   token_ids : device int32 [B]
 *   lut       : device uint8 [V]; lut[v] != 0 sends token id v to the base
 *               (dense) path, 0 to the sparse path.
 *   perm      : device int32 [B], written: the positions b of base-path tokens
 *               in increasing order, then those of sparse-path tokens in
 *               increasing order (a stable partition, bit-exact).
 *   n_dense   : device int32 [1], written: the number of base-path tokens.
 *   dev_status: device int32 [1] or NULL.  If a token id lies outside [0, V)
 *               the kernel ORs 1 into *dev_status and routes that token to the
 *               base path; sats_get_status_word reads it back.
 */
SATS_API sats_status sats_route(const int32_t *token_ids, int B, const uint8_t *lut, int V,
                       int32_t *perm, int32_t *n_dense, int32_t *dev_status, void *stream);

/*
 * sats_mlp_stack -- L decoder MLP blocks on a residual stream:
 *   for l in 0..L-1:  x <- x + MLP_l( RMSNorm(x) * norm_w[l] )
 * with RMSNorm(x) = x / sqrt(mean(x^2) + eps).  Routing (Sec. 3.2) is decided
 * once per token from its id and holds in every block: a base-path token uses
 * the dense MLP (Eq. 1), a sparse-path token the CATS mask with threshold t[l]
 * (Eq. 5).  token_ids == NULL sends every token to the sparse path.
 *   layers    : host array of L layer handles (all with the same H, N)
 *   norm_w    : host array of L device fp32 [H] RMSNorm gains
 *   t         : host fp32 [L], per-layer thresholds (>= 0, not NaN)
 *   token_ids : device int32 [B] or NULL;  lut : device uint8 [V] (V >= 1 when ids given)
 *   x         : device fp32 [B][H], read and overwritten in place.
 *   keep_trace: device uint8 [L][B][N] or NULL; receives each block's keep mask
 *               per token (1 = neuron used), for verification.
 * A token id outside [0, V) is routed to the base path and sets the
 * workspace status word (SATS_EDEVICE from sats_get_error).
 */
SATS_API sats_status sats_mlp_stack(const sats_layer *const *layers, const float *const *norm_w,
                           const float *t, int L, float eps,
                           const int32_t *token_ids, const uint8_t *lut, int V,
                           float *x, int B, uint8_t *keep_trace,
                           void *ws, size_t ws_bytes, void *stream);

/*
 * sats_gate_act -- calibration helper: a = SiLU(x W_gate) (Sec. 2, Eqs. 1-2)
 * for B tokens, the post-gate activations from which thresholds are chosen
 * (Eq. 3 for CATS; candidate set T_l for SATS, Sec. 3.1).
 *   x : device bf16 [B][H];  a : device fp32 [B][N], written.
 */
SATS_API sats_status sats_gate_act(const sats_layer *layer, const void *x, int B, float *a,
                          void *ws, size_t ws_bytes, void *stream);

/*
 * sats_percentile_threshold -- Eq. 3: t = min{t' : F(t') >= k}, F the empirical
 * CDF of |a_i| over n values, i.e. the m-th smallest |a_i| with m = ceil(k n)
 * (k read as a decimal fraction; k*n is taken down by a relative 2^-50 before
 * the ceiling).  k <= 0 gives 0, k > 1 gives +inf.
 *   a      : device fp32 [n] (NaN not allowed)
 *   t_out  : host fp32 [1], written.
 *   ws     : device workspace of at least sats_select_workspace_bytes() bytes.
 * Synchronises `stream` (the result is returned on the host).  Its CTAs (a
 * cooperative launch) wait, bounded, for one another: SATS_ETIMEOUT, with
 * *t_out NaN, if one does not come within 2 s.
 */
SATS_API size_t sats_select_workspace_bytes(void);
SATS_API sats_status sats_percentile_threshold(const float *a, int64_t n, double k, float *t_out,
                                      void *ws, size_t ws_bytes, void *stream);

/*
 * SATS calibration (Sec. 3.1): choose each block's threshold by its local
 * distortion instead of a percentile.
 *
 * sats_rmsnorm -- out[b] = x[b] / sqrt(mean_i x[b][i]^2 + eps) * w, the
 *   pre-MLP normalisation of a decoder block.  x, out: device fp32 [B][H];
 *   w: device fp32 [H].
 *
 * sats_gate_act_f32 -- sats_gate_act for fp32 activations x [B][H].
 *
 * sats_layer_err -- Eq. 6 for K candidate thresholds t (host fp32 [K], each
 *   >= 0) on C calibration inputs x (device fp32 [C][H], the block's MLP
 *   inputs):
 *     err[k] = (1/C) sum_c ||y(x_c) - y~_{t_k}(x_c)||_2 / (||y(x_c)||_2 + eps)
 *     sp[k]  = (1/C) sum_c (neurons with |a| < t_k) / N
 *   y is the dense output (Eq. 1), y~_t the thresholded one (Eqs. 4-5), both
 *   computed by the library's MLP kernels.  err, sp: host double [K].  ws:
 *   device workspace of sats_layer_err_workspace_bytes(H, N, C, K) bytes (an
 *   ordinary workspace for C tokens, 4 C N bytes and at most 512 MiB),
 *   256-byte aligned (no initialisation needed).  Synchronises `stream`.
 *
 * sats_sats_select -- Eqs. 7-10 on the host over a candidate table t, err,
 *   sp (host double [L][K]; every block also has the candidate t = 0 with
 *   error 0 and sparsity 0):
 *     t*_l(b) = max{t in T_l : Err_l(t) <= b}             (Eq. 7)
 *     S(b) = (1/L) sum_l sp_l(t*_l(b))                     (Eqs. 8-9)
 *     b* = argmin_b |S(b) - s_tar|                         (Eq. 10)
 *   over b in {0} and every error in the table, ties to the smaller b.  Block
 *   `guard` (-1 for none) keeps guard_t (sparsity guard_sp) and takes no part
 *   in Eq. 7.  Writes b*, t_out[L] = T*(b*) and S(b*).
 *
 * sats_sats_calibrate -- the whole calibration of an L-block stack, in the
 *   paper's order: (1) the dense stack on the calibration inputs x_cal
 *   (device fp32 [C][H]) gives each block's MLP inputs RMSNorm(x_l) w_l;
 *   (2) coarse candidates: Eq. 3 percentiles of |SiLU(n_l W_gate)| at k/K0,
 *   k = 1..K0-1; (3) Eq. 6 for each; (4) Eqs. 7-10; (5) K1 fine candidates
 *   evenly spaced strictly between the coarse candidates that neighbour each
 *   block's choice (0 below the first, the largest |a| above the last); (6)
 *   Eqs. 6-10 over coarse and fine candidates together.  With guardrail != 0
 *   the last block keeps the CATS threshold (the Eq. 3 percentile at s_tar),
 *   as Sec. 4 does.  Writes t_out (host fp32 [L]), b* and S(b*), and, if all
 *   three are given, the candidate table (host double [L][K0 - 1 + K1]).
 *   ws: sats_sats_workspace_bytes(H, N, C, L, K0, K1) bytes (as sats_layer_err,
 *   4 (L + 1) C H bytes, and at most 1 GiB of values kept between steps 3 and
 *   6), 256-byte aligned.
 *   Synchronises `stream`.
 */
SATS_API sats_status sats_rmsnorm(const float *x, int B, int H, const float *w, float eps, float *out,
                                  void *stream);
SATS_API sats_status sats_gate_act_f32(const sats_layer *layer, const float *x, int B, float *a, void *stream);
SATS_API size_t sats_layer_err_workspace_bytes(int H, int N, int C, int K);
SATS_API sats_status sats_layer_err(const sats_layer *layer, const float *x, int C, const float *t, int K,
                                    float eps, double *err, double *sp, void *ws, size_t ws_bytes, void *stream);
SATS_API sats_status sats_sats_select(const double *t, const double *err, const double *sp, int L, int K,
                                      double s_tar, int guard, double guard_t, double guard_sp, double *b_out,
                                      double *t_out, double *S_out);
SATS_API size_t sats_sats_workspace_bytes(int H, int N, int C, int L, int K0, int K1);
SATS_API sats_status sats_sats_calibrate(const sats_layer *const *layers, const float *const *norm_w, int L,
                                         float eps, const float *x_cal, int C, double s_tar, int K0, int K1,
                                         int guardrail, float err_eps, float *t_out, double *b_out, double *S_out,
                                         double *table_t, double *table_err, double *table_sp, void *ws,
                                         size_t ws_bytes, void *stream);

/*
 * Routing calibration (Sec. 3.2).
 *
 * sats_token_scores -- Eqs. 11-12: for n corpus occurrences (ids: device
 *   int32 [n]; l_base, l_sparse: device fp32 [n], the next-token losses of
 *   the base and sparse paths), d_i = max(0, l_sparse_i - l_base_i) and
 *   score[v] = mean of d_i over the occurrences of v (device fp32 [V]); a
 *   token that never occurs gets +inf (it keeps the base path).  An id
 *   outside [0, V) returns SATS_EDEVICE.  ws: sats_route_calib_workspace_bytes(V)
 *   bytes, 256-byte aligned.  Synchronises `stream`.
 *
 * sats_route_calibrate -- Eq. 14: tau* = argmin_tau |R(tau) - r_tar|, where
 *   R(tau) is the fraction of the m held-out occurrences (heldout_ids: device
 *   int32 [m]) whose score is < tau (routed to the sparse path, Eq. 13); the
 *   candidates are 0, every score of a token occurring in the held-out split,
 *   and +inf, and a tie goes to the smaller tau.  Writes tau* and R(tau*)
 *   (host), and, if lut is given, the routing table lut[v] = score[v] >= tau*
 *   (device uint8 [V]; 1 = base path), as sats_route and sats_mlp_stack take
 *   it.  Synchronises `stream`.
 */
SATS_API size_t sats_route_calib_workspace_bytes(int V);
SATS_API sats_status sats_token_scores(const int32_t *ids, const float *l_base, const float *l_sparse, int64_t n,
                                       int V, float *score, void *ws, size_t ws_bytes, void *stream);
SATS_API sats_status sats_route_calibrate(const float *score, int V, const int32_t *heldout_ids, int64_t m,
                                          double r_tar, float *tau_out, double *R_out, uint8_t *lut, void *ws,
                                          size_t ws_bytes, void *stream);

/*
 * Vocabulary operators: rows of logits, on either side of the token routing.
 * The token ids that sats_route looks up are drawn from logits, and the losses
 * that sats_token_scores takes are losses of logits; the paper leaves both to
 * the model around the method.
 *
 * In all of them logits is a device array of rows of V elements (bf16, or fp32
 * in the _f32 calls), row r starting at element r * ld (ld >= V; what lies
 * between the rows is not read).  A pointer needs the alignment of its elements
 * only.  The calls need no workspace, and what they write does not depend on the
 * order in which their threads run.  In sats_distill_loss_grad the CTAs of a row
 * wait, bounded, for one another's sums: if one gives up, dev_status tells
 * (SATS_ETIMEOUT from sats_get_status_word), and the loss and gradient of that
 * row and of the rows that these CTAs serve after it are NaN wherever they are
 * not right.  V up to 2^31 - 65 and 2^28 - 1 rows (else
 * SATS_ESHAPE); no rows: nothing is done.
 *
 * sats_top_logits -- the K largest logits of each row, as a teacher hands them
 *   over: values (device fp32 [T][K]) in descending order, ties by the lower
 *   index first, and their indices idx (device int32 [T][K]).  -inf and NaN
 *   are never selected: a row with fewer other elements gets -inf and index -1
 *   in the places left (an absent entry, for the calls below).  1 <= K <= V;
 *   K up to 1024 (else SATS_ESHAPE).
 *
 * sats_distill_loss -- the loss of a row z against a teacher's top logits and
 *   a label, with temperature tau and share alpha:
 *     q = softmax over the row's entries of top_val / tau
 *     KD = tau^2 sum_k q_k (log q_k - log softmax(z / tau)[top_idx_k])
 *     CE = log sum_j exp(z_j) - z[label]
 *     loss = alpha KD + (1 - alpha) CE
 *   With alpha 0 (K may be 0 then) it is the next-token loss that
 *   sats_token_scores takes for the base and the sparse path.
 *   top_idx, top_val : device int32 and fp32 [T][K] (K 0 to 1024; NULL if 0).  An
 *                index below 0 is an absent entry, and so is one with the value
 *                -inf; a row without any has KD = 0.  An index may occur twice.
 *                A NaN or +inf value makes the row's loss NaN.
 *   labels     : device int32 [T], or NULL for no CE term (CE = 0).  A label
 *                below 0 makes its row an ignored one: nothing of it is read,
 *                its loss, lse and gradient are 0.
 *   tau, alpha : 2^-10 <= tau <= 2^10, 0 <= alpha <= 1; at least one of the two terms
 *                must be there (else SATS_EINVAL).
 *   loss       : device fp32 [T], written.
 *   lse        : device fp32 [T][2] or NULL; log sum_j exp(z_j / tau) and
 *                log sum_j exp(z_j), for sats_distill_grad.
 *   dev_status : device int32 [1] or NULL.  An index or label >= V sets it
 *                (SATS_EDEVICE from sats_get_status_word); the entry is then
 *                absent, the row an ignored one.
 *   A row with a NaN or +inf logit, or with none above -inf, has the loss NaN if a
 *   term counts there (entries, with alpha > 0; a label, with alpha < 1), else 0.
 *   Logits are divided by tau in fp32: where tau < 1, what of them passes fp32's
 *   range counts as an infinity in lse.  A probability below 2^-126 may count as 0.
 *
 * sats_distill_grad -- its backward pass:
 *     dlogits_j = g (alpha tau (softmax(z / tau)_j - sum_{k: top_idx_k = j} q_k)
 *                    + (1 - alpha) (softmax(z)_j - [j = label]))
 *   from the same arguments and the lse that sats_distill_loss wrote, whose
 *   rounding it inherits: 2^-24 |lse| relative.  Of a row whose loss its logits
 *   make NaN it is NaN everywhere; if g is 0 or no term counts, 0 but for NaN at
 *   the NaN and +inf logits.  A NaN or +inf value makes it NaN at the row's
 *   entries.
 *   g          : device fp32 [T], the gradient of each row's loss, or NULL for 1.
 *   dlogits    : device, the logits' type, rows of V elements ld_d >= V apart,
 *                written (each value rounded once).  It may be the logits
 *                themselves (the same pointer and row stride), or lie between
 *                their rows (the same row stride); any other overlap of the two
 *                areas returns SATS_EINVAL.
 *
 * sats_distill_loss_grad -- both in one pass over the logits, for a caller who
 *   knows g beforehand (a mean over the batch): loss and dlogits as above.
 *
 * sats_sample -- draws one token from each of B rows, from given random numbers.
 *   With z the row, T its temperature and w_i = exp((z_i - max z) / T):
 *     top-k: the k largest logits are kept (ties: the lower index first);
 *     top-p: of these the shortest run of the largest (ties as before) whose
 *            share of their mass sum w reaches p, one at least;
 *     min-p: of these the ones with w_i >= min_p;
 *   the token is the first kept one, in the vocabulary's order, at which the
 *   running sum of w exceeds u times its total over the kept ones.
 *   temperature, top_k, top_p, min_p : device fp32 / int32 / fp32 / fp32 [B],
 *                or NULL for 1, off, off, off.  T >= 0 and finite, 0: the largest
 *                logit (the lowest index that has it); above 0 and below 1e-30: one
 *                of the largest, all alike.  top_k <= 0 or >= V is off,
 *                top_p >= 1 is off, top_p <= 0 keeps one, min_p <= 0 is off,
 *                min_p <= 1.
 *   u          : device fp32 [B], random numbers in [0, 1).
 *   ids        : device int32 [B], written.
 *   logprob    : device fp32 [B] or NULL; the log of the drawn token's share of
 *                the kept mass.
 *   n_kept     : device int32 [B] or NULL; how many tokens were kept.
 *   -inf and NaN logits are never kept; where there are no others, the id is -1,
 *   logprob -inf and n_kept 0.  If the largest logit is +inf, all that have it
 *   weigh the same and the others nothing.  A setting outside its range (a NaN,
 *   T < 0, min_p > 1, u outside [0, 1)) gives the id -1, logprob NaN and n_kept 0 and
 *   sets *dev_status (device int32 [1] or NULL; SATS_EDEVICE).
 *   The weights are whole multiples of 2^-43 of the largest (of 2^-(62 - bits of V)
 *   from V = 2^18 on), right to about 35 bits of themselves (to fewer above
 *   T = 2^110, whose inverse has fewer in fp32); their sums are exact.
 */
SATS_API sats_status sats_top_logits(const void *logits, int64_t ld, int T, int V, int K, float *values, int32_t *idx,
                                     void *stream);
SATS_API sats_status sats_top_logits_f32(const float *logits, int64_t ld, int T, int V, int K, float *values,
                                         int32_t *idx, void *stream);
SATS_API sats_status sats_distill_loss(const void *logits, int64_t ld, int T, int V, const int32_t *top_idx,
                                       const float *top_val, int K, const int32_t *labels, float tau, float alpha,
                                       float *loss, float *lse, int32_t *dev_status, void *stream);
SATS_API sats_status sats_distill_loss_f32(const float *logits, int64_t ld, int T, int V, const int32_t *top_idx,
                                           const float *top_val, int K, const int32_t *labels, float tau, float alpha,
                                           float *loss, float *lse, int32_t *dev_status, void *stream);
SATS_API sats_status sats_distill_grad(const void *logits, int64_t ld, int T, int V, const int32_t *top_idx,
                                       const float *top_val, int K, const int32_t *labels, float tau, float alpha,
                                       const float *lse, const float *g, void *dlogits, int64_t ld_d,
                                       int32_t *dev_status, void *stream);
SATS_API sats_status sats_distill_grad_f32(const float *logits, int64_t ld, int T, int V, const int32_t *top_idx,
                                           const float *top_val, int K, const int32_t *labels, float tau, float alpha,
                                           const float *lse, const float *g, float *dlogits, int64_t ld_d,
                                           int32_t *dev_status, void *stream);
SATS_API sats_status sats_distill_loss_grad(const void *logits, int64_t ld, int T, int V, const int32_t *top_idx,
                                            const float *top_val, int K, const int32_t *labels, float tau,
                                            float alpha, const float *g, float *loss, void *dlogits, int64_t ld_d,
                                            int32_t *dev_status, void *stream);
SATS_API sats_status sats_distill_loss_grad_f32(const float *logits, int64_t ld, int T, int V, const int32_t *top_idx,
                                                const float *top_val, int K, const int32_t *labels, float tau,
                                                float alpha, const float *g, float *loss, float *dlogits, int64_t ld_d,
                                                int32_t *dev_status, void *stream);
SATS_API sats_status sats_sample(const void *logits, int64_t ld, int B, int V, const float *temperature,
                                 const int32_t *top_k, const float *top_p, const float *min_p, const float *u,
                                 int32_t *ids, float *logprob, int32_t *n_kept, int32_t *dev_status, void *stream);
SATS_API sats_status sats_sample_f32(const float *logits, int64_t ld, int B, int V, const float *temperature,
                                     const int32_t *top_k, const float *top_p, const float *min_p, const float *u,
                                     int32_t *ids, float *logprob, int32_t *n_kept, int32_t *dev_status, void *stream);

/*
 * Adjusted logits: what lies between the model's logits and sats_sample, and its gradient.
 * logits, out, dout, dlogits are rows as in the vocabulary operators above (any alignment of whole
 * elements, row strides of at least V elements).  The calls need no workspace, and what they write does not depend on the
 * order in which their threads run.  V up to 2^31 - 65, 2^28 - 1 rows, L below 2^30 (else SATS_ESHAPE).
 *
 * sats_adjust_logits -- for each of B rows z with its history of token ids:
 *     z_v <- z_v > 0 ? z_v / r : z_v r      where v occurs in the history
 *     z_v <- z_v - f c_v - p                where v occurs c_v > 0 times in the generated part of it
 *     z_v <- z_v + bias_v
 *     z_v <- -inf                           where the mask does not allow v
 *   in fp32, rounded once.
 *   hist       : device int32, row b at b * ld_hist, L ids at most (ld_hist 0: all rows share one; rows may overlap), or
 *                NULL with L 0 (then hist_len and n_prompt are not looked at).  Ids below 0 are absent.
 *   hist_len   : device int32 [B], how many ids of its row count (NULL: L).
 *   n_prompt   : device int32 [B] or NULL for 0: the first n_prompt ids are the prompt, the others are generated.
 *   repetition, presence, frequency : r, p, f, device fp32 [B] or NULL for off (1, 0, 0).  r > 0, all finite.
 *                The history of a row whose three are off is not read, of another one no more than the ids that count.
 *   bias_idx, bias_val : device int32 and fp32 [B][M] (M up to 1024, else SATS_ESHAPE; NULL if 0).  An index below 0 is an
 *                absent entry; of entries with the same index the last one counts.  -inf makes the logit -inf.
 *   mask       : device int32 words of 32 tokens each (bit v mod 32 of word v / 32: v is allowed), row i at i * ld_mask
 *                (ld_mask >= ceil(V / 32)), n_masks rows; or NULL.
 *                A pointer to int32 or fp32 values, the mask's too, that is not 4-byte aligned: SATS_EINVAL.
 *   mask_row   : device int32 [B], the mask of each row; below 0: none.  NULL: mask b for row b (n_masks >= B).
 *   out        : the logits' type; the logits themselves (same pointer and stride), or between their rows (same
 *                stride), or elsewhere (another overlap: SATS_EINVAL).  In place only the logits that change are
 *                read and written; a row's ids are looked at once for every 1024 to 16384 of its V logits all the same.
 *   dev_status : device int32 [1] or NULL.  Set (SATS_EDEVICE) by a setting outside its range, which is off then; an id
 *                or index >= V, a NaN or +inf bias, which are absent then; a hist_len outside [0, L], which is taken
 *                as the nearer of the two (so is n_prompt, without being noted); a mask_row >= n_masks, which is none.
 *   A NaN logit stays NaN unless it becomes -inf.
 *
 * sats_adjust_logits_grad -- its backward pass: dlogits_v = dout_v times 0 where the mask does not allow v (also where
 *   dout is not finite), 1 / r or r where v occurs in the history (r at z_v = 0), else 1.  The biases and the other two
 *   penalties are constants here.  logits: what sats_adjust_logits was given, read only at the tokens of the history.
 *   dlogits may be dout (same pointer and stride), or lie between the rows of dout or the logits; not the logits.
 */
SATS_API sats_status sats_adjust_logits(const void *logits, int64_t ld, int B, int V, const int32_t *hist,
                                        int64_t ld_hist, int L, const int32_t *hist_len, const int32_t *n_prompt,
                                        const float *repetition, const float *presence, const float *frequency,
                                        const int32_t *bias_idx, const float *bias_val, int M, const void *mask,
                                        int64_t ld_mask, int n_masks, const int32_t *mask_row, void *out,
                                        int64_t ld_out, int32_t *dev_status, void *stream);
SATS_API sats_status sats_adjust_logits_f32(const float *logits, int64_t ld, int B, int V, const int32_t *hist,
                                            int64_t ld_hist, int L, const int32_t *hist_len, const int32_t *n_prompt,
                                            const float *repetition, const float *presence, const float *frequency,
                                            const int32_t *bias_idx, const float *bias_val, int M, const void *mask,
                                            int64_t ld_mask, int n_masks, const int32_t *mask_row, float *out,
                                            int64_t ld_out, int32_t *dev_status, void *stream);
SATS_API sats_status sats_adjust_logits_grad(const void *logits, int64_t ld, int B, int V, const int32_t *hist,
                                             int64_t ld_hist, int L, const int32_t *hist_len, const float *repetition,
                                             const void *mask, int64_t ld_mask, int n_masks, const int32_t *mask_row,
                                             const void *dout, int64_t ld_dout, void *dlogits, int64_t ld_d,
                                             int32_t *dev_status, void *stream);
SATS_API sats_status sats_adjust_logits_grad_f32(const float *logits, int64_t ld, int B, int V, const int32_t *hist,
                                                 int64_t ld_hist, int L, const int32_t *hist_len,
                                                 const float *repetition, const void *mask, int64_t ld_mask,
                                                 int n_masks, const int32_t *mask_row, const float *dout,
                                                 int64_t ld_dout, float *dlogits, int64_t ld_d, int32_t *dev_status,
                                                 void *stream);

/*
 * 4-bit weights with group scales: a matrix W [K][N] (y = x W; the vocabulary head, a projection) as whole numbers
 * from -8 to 7 times a scale for every G consecutive k of a column:
 *     W[k][n] = scales[k / G][n] * q[k][n]
 *   codes  : uint8 [K / 2][N]; byte (i, n) holds q[2i][n] in its low and q[2i + 1][n] in its high half (two's complement)
 *   scales : bf16 [ceil(K / G)][N], any sign; one that is not finite makes its column of y NaN.
 * K a multiple of 8 and 8 <= K <= 65536; 1 <= N <= 2^24; G 32, 64 or 128 (else SATS_ESHAPE).
 *
 * sats_q4_quantize -- codes and scales (device, written) of a bf16 matrix W (device [K][N], rows ld >= N elements
 *   apart): over each group s = amax / 7 rounded to bf16, q = w / s rounded half to even, within [-7, 7].  A group with a NaN or an
 *   infinity gets the scale NaN.
 * sats_q4_dequantize -- what codes and scales stand for: values device fp32 [K][N], exact.
 *
 * sats_q4_create -- packs codes and scales (device) into a handle, which owns its device memory: with K and N rounded
 *   up to multiples of 128, K N / 2 bytes, 2 K N / G for the scales and 4 per column. Runs on `stream` and synchronises
 *   it; the caller may then free both. Within a column scales are kept to 8 significant bits from its largest one down
 *   to 2^-21 of it, below as multiples of 2^-28 of it. It belongs to the device that is current then; products with
 *   another current device are refused (SATS_EINVAL).
 * sats_q4_destroy frees it (synchronises its device first); sats_q4_shape reads back K, N, G (each may be NULL).
 *
 * sats_q4_matmul -- y = x W for B tokens (up to 2^20): x device bf16 [B][K] (fp32 in the _f32 call), y device [B][N],
 *   rows ld_y >= N elements apart, fp32 if y_f32 is not 0, else bf16; both need the alignment of their elements only.
 *   x, y (its rows) and what the call needs of ws must not overlap (SATS_EINVAL). The tensor cores multiply the weights
 *   exactly and the activations to 11 (bf16: all of its 8) or 22 (fp32) significant bits, absolute 2^-39 (2^-50) of a
 *   token's largest. Sums are rounded to fp32 every 128 products, whatever the number of tokens; on the way there the
 *   tensor cores cut them in 8 steps, each to no fewer than 22 bits. So a result is off by at most 2^-18 + (K / 128 +
 *   2) 2^-24 of its sum |x| |W| (fp32 activations 2^-22 more), before it is rounded to bf16 where that is asked for;
 *   observed: 2^-19.8 where all terms have one sign, so that the cuts add up; 1e-7 to 4e-7 of the norm. Where K is
 *   divided among CTAs the parts are fp32 numbers of the result's own size: one that passes fp32's range makes the
 *   result an infinity. The same call gives the same bits every time; another batch size may divide K otherwise and
 *   give a token's others.
 *   ws: device, 256-byte aligned, of sats_q4_workspace_bytes(K, N, B) bytes or more (0: shape out of range), zero-filled
 *   once before first use (sats_workspace_init), left ready for the next call, of any batch and weights that fit; calls
 *   that share one must not overlap on the GPU.  A bounded wait that gives up leaves y incomplete, sats_get_error(ws)
 *   says SATS_ETIMEOUT, and the workspace has to be zero-filled again.  As the decode kernel the call's own kernels
 *   may begin before the kernel before them in the stream has ended, reading the weights only until it has.
 */
SATS_API sats_status sats_q4_quantize(const void *W, int64_t ld, int K, int N, int G, uint8_t *codes, void *scales,
                                      void *stream);
SATS_API sats_status sats_q4_dequantize(const uint8_t *codes, const void *scales, int K, int N, int G, float *values,
                                        void *stream);
SATS_API sats_status sats_q4_create(const uint8_t *codes, const void *scales, int K, int N, int G, void *stream,
                                    sats_q4 **out);
SATS_API sats_status sats_q4_destroy(sats_q4 *w);
SATS_API sats_status sats_q4_shape(const sats_q4 *w, int *K, int *N, int *G);
SATS_API size_t sats_q4_workspace_bytes(int K, int N, int B);
SATS_API sats_status sats_q4_matmul(const sats_q4 *w, const void *x, int B, void *y, int64_t ld_y, int y_f32, void *ws,
                                    size_t ws_bytes, void *stream);
SATS_API sats_status sats_q4_matmul_f32(const sats_q4 *w, const float *x, int B, void *y, int64_t ld_y, int y_f32,
                                        void *ws, size_t ws_bytes, void *stream);

/*
 * sats_selftest_wait_timeout -- exercises the failure path of the device-side
 * waits without a fault: one small kernel runs the library's bounded waits on
 * conditions nothing satisfies (an mbarrier phase no thread completes, a
 * workspace counter no CTA raises).  Each gives up after its time limit (2 s)
 * and records a timeout in the workspace status word, so a following
 * sats_get_error returns SATS_ETIMEOUT (and clears it).  Takes about 4 s;
 * the workspace and the device stay usable.  ws: a workspace of any layer
 * shape (at least 256 bytes), not in use by another call.
 */
SATS_API sats_status sats_selftest_wait_timeout(void *ws, size_t ws_bytes, void *stream);

/*
 * sats_selftest_select_timeout -- the same for sats_percentile_threshold: its
 * selection over a (device fp32 [n], n >= 1) at k = 1, waiting for one CTA
 * more than there are.  Returns SATS_ETIMEOUT after about 2 s, with *t_out NaN;
 * arguments and workspace as there.
 */
SATS_API sats_status sats_selftest_select_timeout(const float *a, int64_t n, float *t_out, void *ws,
                                                  size_t ws_bytes, void *stream);

/*
 * sats_selftest_distill_timeout -- the same for sats_distill_loss_grad: a call
 * on bf16 logits with labels alone (tau 1, alpha 0, g NULL; arguments as there,
 * 0 <= row < T), in which one CTA of the given row does not get another's sums.
 * Where a row has more than one CTA (rows beyond 72 KB, or few of them), the
 * wait for them gives up after 2 s and those that depend on it after 2 s more;
 * dev_status says SATS_ETIMEOUT.
 */
SATS_API sats_status sats_selftest_distill_timeout(const void *logits, int64_t ld, int T, int V, const int32_t *labels,
                                                   float *loss, void *dlogits, int64_t ld_d, int row,
                                                   int32_t *dev_status, void *stream);

/*
 * sats_get_error -- synchronises `stream`, reads the status word in the
 * workspace, clears it, and returns SATS_OK, SATS_EDEVICE (bad token id) or
 * SATS_ETIMEOUT (a device wait gave up).
 */
SATS_API sats_status sats_get_error(void *ws, size_t ws_bytes, void *stream);

/* Same for a caller-owned status word (as passed to sats_route). */
SATS_API sats_status sats_get_status_word(int32_t *dev_status, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* SATS_H */
