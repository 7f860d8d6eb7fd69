/*
 * wersa.h -- C ABI of the WERSA attention hot path for AMD MI355X (gfx950).
 *
 * WERSA (Wavelet-Enhanced Random Spectral Attention) per (batch, head) slice, with
 * Q, K, V in R^{n x d} (paper Section 3.1, steps 3-8):
 *
 *   qbar   = mean over the n rows of Q                                   (step 4, Q'_avg)
 *   F_i    = sigmoid(W_g[h] qbar + b_g[h])_i * omega_i,  i = 0..L        (step 4, F_i)
 *   X_F    = W^-1( F (.) W X )  for X in {Q, K}; W = L-level Haar DWT    (steps 3, 5, 6)
 *            band 0 = finest detail d_1 ... band L-1 = d_L, band L = approximation a_L
 *            (return order of Algorithm 2's DWT); the same F gates Q and K
 *   Phi_X  = ReLU( X_F Omega / sigma_eff ) / sqrt(m),  sigma_eff = max(sigma, bw_floor)
 *                                                    (step 7; Algorithm 1 projection lines)
 *   S      = Phi_K^T V  (m x d),   z = Phi_K^T 1  (m)                    (step 8 numerator/denominator)
 *   O      = (Phi_Q S) / (Phi_Q z + eps)                                 (step 8, attention equation)
 *
 * wersa_backward returns the gradients of a scalar loss with respect to Q, K, V, W_g, b_g,
 * omega and sigma given dO = d loss / d O (the paper states no backward; it is the derivative
 * of the forward above).
 *
 * Conventions
 *   - Every data pointer is a DEVICE pointer owned by the caller. The library allocates
 *     nothing, frees nothing and never synchronises: work is enqueued on `hip_stream`
 *     (a hipStream_t passed as void*, NULL = the default stream) and the call returns.
 *   - Tensors q, k, v, out, dout, dq, dk, dv share one layout: element (b, h, t, j) lives at
 *     b*stride_b + h*stride_h + t*stride_n + j (strides in elements, j contiguous).
 *   - omega_rf (the random matrix Omega) is d x m row-major in the tensor dtype.
 *   - Parameters and their gradients are float32: gate_w [H][L+1][d], gate_b [H][L+1],
 *     scale_w [L+1] (the per-scale weights omega), sigma [1].
 *   - Gradients are overwritten, not accumulated. dgate_w, dgate_b, dscale_w, dsigma may each
 *     be NULL to skip that output.
 *   - `saved` is written by wersa_forward and read by wersa_backward (wersa_saved_bytes).
 *     `workspace` is scratch, at least wersa_workspace_bytes; both 256-byte aligned.
 *   - All argument validation happens before anything is enqueued; on error nothing is
 *     launched. No exception or abort crosses the boundary.
 *   - No mutable global state apart from the optional profiling switch below: calls on
 *     different streams with different buffers may overlap.
 *   - Results are deterministic: reductions use fixed-order two-pass sums, no float atomics.
 */
#ifndef WERSA_H
#define WERSA_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  WERSA_OK = 0,
  WERSA_ERR_INVALID_ARG = 1, /* NULL pointer, non-positive size, bad stride or enum       */
  WERSA_ERR_UNSUPPORTED = 2, /* valid problem outside the implemented range (see desc)    */
  WERSA_ERR_WORKSPACE = 3,   /* workspace_bytes too small or misaligned                    */
  WERSA_ERR_LAUNCH = 4       /* the HIP runtime refused a launch                           */
} wersa_status;

typedef enum { WERSA_F32 = 0, WERSA_BF16 = 1 } wersa_dtype;

/* desc.flags bits. By default the library picks the MFMA path (bf16 storage, fp16/bf16 matrix
 * cores, float32 accumulation) when the shape allows it: dtype bf16, d in {64, 128},
 * m % 128 == 0, strides multiples of 8 elements (any n, any L <= 20);
 * otherwise the generic path:
 * float32 arithmetic throughout (contractions on the bf16 matrix cores with every float32 operand as
 * the sum of three bf16 values for d <= 128, float32 matrix instructions above, with few rows, and where only these
 * keep the forward's workspace within wersa_static_scratch_bytes()).
 * WERSA_FLAG_GENERIC_PATH forces the generic path. */
#define WERSA_FLAG_GENERIC_PATH 1
/* Separate random matrices for the query and the key side (Algorithm 1 draws W_Q^rand and
 * W_K^rand independently; Section 3.1 step 7 uses one): omega_rf then holds two d x m row-major
 * matrices back to back, the query-side one first. */
#define WERSA_FLAG_SEPARATE_OMEGA 2
/* Gate pooled over heads (Algorithm 1: the pooled queries of all heads of a batch element are
 * concatenated and go through one linear map, giving one filter per batch element):
 * logits_i = sum_h (gate_w[h][i] . qbar_h + gate_b[h][i]), F = sigmoid(logits) * scale_w for every
 * head of that batch element. Parameter shapes are unchanged (gate_w read as the (L+1) x (H*d)
 * map in head blocks). Default (Section 3.1 step 4): each head gates itself. */
#define WERSA_FLAG_POOLED_GATE 4
/* Output stage of Algorithm 1: O = LayerNorm(phi(Q_F) (phi(K_F)^T V)) over the d columns of each
 * row (no affine parameters, biased variance, desc.eps inside the square root) in place of
 * Section 3.1's division by the normaliser. The saved per-row value is then 1 / sqrt(var + eps). */
#define WERSA_FLAG_LAYERNORM 8

/*
 * Problem descriptor (host memory, read during the call only).
 * Supported range: B, H >= 1 with B * H <= 1023 (the slices are one grid dimension of every
 * launch, shared with the split of n; larger batches are to be split over calls);
 * 1 <= n <= 2^22; 0 <= L <= 20; d % 16 == 0, 16 <= d <= 256; m % 16 == 0, 16 <= m <= 4096.
 * Anything else that is otherwise well formed returns WERSA_ERR_UNSUPPORTED.
 * MFMA path only: the filtered Q and K enter the random projection (step 7) rounded to fp16, after
 * a power-of-two scale chosen per (batch, head) slice from max|Q| and the filter of that slice
 * (ReLU is positively homogeneous, so the scale drops out exactly); inputs, bandwidth and per-scale
 * weights of any magnitude are fine as long as the filtered K of a slice stays below about 2^11
 * times the bound on its filtered Q (beyond that the fp16 operands overflow: take
 * WERSA_FLAG_GENERIC_PATH).  The block entry points take the same maxima from the epilogue of their
 * W^Q product (when n % 128 != 0 or L > 6 the core pools, and scales, by itself).
 * MFMA path only: q, k, v, omega_rf, out, dout, dq, dk, dv must be 16-byte aligned (their rows
 * are read and written in 16-byte pieces); a misaligned pointer returns WERSA_ERR_INVALID_ARG
 * before anything is enqueued (WERSA_FLAG_GENERIC_PATH takes any element-aligned pointer).
 * Any n is accepted: the Haar filter is local to aligned blocks of 2^L rows, so Algorithm 2's
 * zero padding to the next power of two and the trim after the inverse are the same as reading
 * the rows past n of the last block as zeros and not writing them (done in-kernel; the pooled
 * query averages the n real rows). L > 6 (blocks longer than one 64-row tile): six levels run
 * inside the tiles, the rest on per-tile sums.
 */
typedef struct {
  int32_t B, H, n, d, L, m;
  int32_t dtype;         /* wersa_dtype of q, k, v, omega_rf, out, dout, dq, dk, dv        */
  float eps;             /* epsilon of the normaliser (Section 3.1 step 8)                  */
  float bw_floor;        /* floor of the bandwidth (Algorithm 1: bw = max(beta, floor))     */
  int64_t stride_b, stride_h, stride_n;
  int32_t flags;         /* 0 or WERSA_FLAG_* bits                                          */
} wersa_desc;

/* Bytes of scratch needed by wersa_forward (for_backward == 0) or wersa_backward (!= 0).
 * Returns 0 if the descriptor is invalid or unsupported. */
size_t wersa_workspace_bytes(const wersa_desc *desc, int for_backward);

/* Bytes of the buffer that carries S, z, qbar, the gate activations, F and the normaliser D
 * from forward to backward (and, of small float32-arithmetic problems and of bf16 ones with d = 128, the filtered Q and
 * K). Returns 0 if the descriptor is invalid or unsupported. */
size_t wersa_saved_bytes(const wersa_desc *desc);

/* Forward pass (Section 3.1 steps 3-8). Writes out (B,H,n,d) and saved. */
wersa_status wersa_forward(const wersa_desc *desc, const void *q, const void *k, const void *v,
                           const void *omega_rf, const float *sigma, const float *gate_w,
                           const float *gate_b, const float *scale_w, void *out, void *saved,
                           void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * wersa_forward for callers that cannot allocate device memory (code under HIP graph capture,
 * tight serving loops, harnesses that forbid hipMalloc): the same computation with the workspace
 * taken from a scratch array built into the library (device memory, wersa_static_scratch_bytes()
 * = 40 MiB per GPU, held from the first use until the process ends).  The caller still passes
 * inputs, `out` and `saved`; the call allocates nothing and never synchronises.  A problem whose
 * wersa_workspace_bytes(desc, 0) exceeds the scratch returns WERSA_ERR_WORKSPACE before anything is
 * enqueued (the MFMA-path forward needs 17-35 MiB at the benchmark shapes, so those fit; deeper
 * transforms than six levels at long n and large generic-path problems do not).  Every call on a
 * GPU shares that GPU's array, whose contents are scratch (nothing in it needs to start at zero):
 * calls that overlap in time on one GPU, on any streams, race; calls on different GPUs do not.
 * The device that is current at the call must be the one that holds the tensors.
 */
size_t wersa_static_scratch_bytes(void);
wersa_status wersa_forward_static(const wersa_desc *desc, const void *q, const void *k, const void *v,
                                  const void *omega_rf, const float *sigma, const float *gate_w,
                                  const float *gate_b, const float *scale_w, void *out, void *saved,
                                  void *hip_stream);

/* Backward pass: derivative of wersa_forward. `out` and `saved` are those of the matching
 * forward call on the same inputs. */
wersa_status wersa_backward(const wersa_desc *desc, const void *q, const void *k, const void *v,
                            const void *omega_rf, const float *sigma, const float *gate_w,
                            const float *gate_b, const float *scale_w, const void *out,
                            const void *dout, const void *saved, void *dq, void *dk, void *dv,
                            float *dgate_w, float *dgate_b, float *dscale_w, float *dsigma,
                            void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Stage entry point: the gated Haar filter alone, X_F = W^-1(F (.) W X) (Section 3.1 steps
 * 3, 5, 6; Appendix A equations) for one tensor x laid out like q, with per-slice filter
 * coefficients filt [B*H][L+1] (float32, device). Output xf has the same layout and dtype.
 * It takes no workspace and covers L <= 6; a deeper transform returns WERSA_ERR_UNSUPPORTED here
 * (wersa_haar_filter_ws takes it).
 */
wersa_status wersa_haar_filter(const wersa_desc *desc, const void *x, const float *filt,
                               void *xf, void *hip_stream);

/*
 * The same stage for every L the library takes (Appendix A: L = O(log n)). Levels above 6 run
 * on the approximation coefficients of the 64-row tiles, which live in `workspace` (device
 * memory owned by the caller, 256-byte aligned, at least wersa_haar_filter_workspace_bytes(desc)
 * bytes; 0 bytes and a NULL pointer are fine for L <= 6). Contents of the workspace are scratch.
 * Errors as for wersa_forward; a workspace that is too small or misaligned returns
 * WERSA_ERR_WORKSPACE before anything is enqueued.
 */
size_t wersa_haar_filter_workspace_bytes(const wersa_desc *desc);
wersa_status wersa_haar_filter_ws(const wersa_desc *desc, const void *x, const float *filt,
                                  void *xf, void *workspace, size_t workspace_bytes,
                                  void *hip_stream);

/*
 * Attention block around the core (Section 3.1 steps 1-2: Q' = X W^Q, K' = X W^K, V' = X W^V,
 * split into H heads of width d; Algorithm 1's last line: merged heads times W_out):
 *   Y = merge_heads( WERSA( split(X W^Q), split(X W^K), split(X W^V) ) ) W^out
 * x, y, dy, dx are dense (B, n, hidden) with hidden = H*d in bf16; head h owns columns
 * [h*d, (h+1)*d) and is addressed by stride (nothing is transposed); the four weights are
 * hidden x hidden row-major [in][out] in bf16; their gradients are float32 [in][out],
 * overwritten. The stride fields of desc are ignored. Supported: dtype bf16, hidden % 256 == 0,
 * (B*n) % 256 == 0, and the core's own limits; otherwise WERSA_ERR_UNSUPPORTED.
 * `saved` (wersa_block_saved_bytes) carries Q', K', V', the merged head outputs A and the
 * core's saved buffer from forward to backward; `workspace` (wersa_block_workspace_bytes) is
 * scratch. The other conventions are those of wersa_forward / wersa_backward; the core
 * parameter gradients may be NULL, the weight gradients may not.
 */
size_t wersa_block_workspace_bytes(const wersa_desc *desc, int for_backward);
size_t wersa_block_saved_bytes(const wersa_desc *desc);

wersa_status wersa_block_forward(const wersa_desc *desc, const void *x, const void *wq,
                                 const void *wk, const void *wv, const void *wo,
                                 const void *omega_rf, const float *sigma, const float *gate_w,
                                 const float *gate_b, const float *scale_w, void *y, void *saved,
                                 void *workspace, size_t workspace_bytes, void *hip_stream);

wersa_status wersa_block_backward(const wersa_desc *desc, const void *x, const void *wq,
                                  const void *wk, const void *wv, const void *wo,
                                  const void *omega_rf, const float *sigma, const float *gate_w,
                                  const float *gate_b, const float *scale_w, const void *dy,
                                  const void *saved, void *dx, float *dwq, float *dwk, float *dwv,
                                  float *dwo, float *dgate_w, float *dgate_b, float *dscale_w,
                                  float *dsigma, void *workspace, size_t workspace_bytes,
                                  void *hip_stream);

/* Byte offsets of the pieces inside the block's `saved`, for tests and tools: which = 0 Q',
 * 1 K', 2 V', 3 A (each bf16 (B, n, hidden)), 4 the core's saved buffer. -1 on a bad argument. */
int64_t wersa_block_saved_offset(const wersa_desc *desc, int which);

/* Byte offsets inside the backward `workspace` of the intermediate gradients left there by
 * wersa_block_backward, for tests and tools: which = 0 dA, 1 dQ', 2 dK', 3 dV' (each bf16
 * (B, n, hidden)). -1 on a bad argument. */
int64_t wersa_block_workspace_offset(const wersa_desc *desc, int which);

/*
 * Causal linear attention with a decay for each head (the causal counterpart of step 8 without a normaliser, for decoders):
 *   S_t = lambda_h S_{t-1} + k_t v_t^T  (dk x dv, float32),  o_t = scale q_t^T S_t,  lambda_h = exp(log_decay[h])
 * over a whole sequence (wersa_decay_forward), its derivative (wersa_decay_backward), and one token at a time on a
 * cache of states (wersa_decay_step).  q and k are (B, H, n, dk), v and out (B, H, n, dv), each at strides of its own
 * (batch, head, row; in elements; columns contiguous); dout is laid out like out.  Any element-aligned pointer is taken.  Rows do
 * not overlap: a row's stride is at least the width, and at most 2^24; with n = 1 it is not read.  Sequences and heads of what is
 * only read may overlap (strides above 0); in out, dq, dk and dv each dimension begins behind what those of smaller strides take.
 *   packed   0: B sequences of n rows each; offsets is NULL.
 *            1: B sequences of any lengths (zero among them) one behind the other in tensors with one batch entry of n
 *               rows: sequence b is rows offsets[b] .. offsets[b + 1] - 1 (B + 1 device integers that do not decrease; the
 *               batch strides are not read).  Offsets are clamped to 0 .. n on the device.  Rows of no sequence,
 *            before the first one's or behind the last one's, are not read; the forward leaves them in out as they are, or with
 *            clear = 1 writes zeros to them; in dq, dk and dv they are zeros.
 *   log_decay  float32 [H], at most 0 for a state that stays bounded; -inf is a decay of zero.  A fixed parameter: it
 *            has no gradient.
 *   states   float32 [state_slots][H][dk][dv], contiguous, 16-byte aligned.  initial_state NULL: zeros; final_state
 *            NULL: not wanted; the two may be the same buffer.  slots NULL: sequence b has state b.  Otherwise sequence b has
 *            state slots[b] (device integers, no two alike); one below 0 or from state_slots on has none: its initial state is
 *            zero, its final state is not written, and wersa_decay_step gives it zeros.
 *   saved    what the forward leaves for the backward (wersa_decay_saved_bytes, 256-byte aligned); NULL: no backward
 *            follows, and the workspace takes it.  A forward that is given `saved` needs no workspace.
 * wersa_decay_backward: the gradients of a scalar loss given those with respect to out and (dfinal_state, by sequence, may be
 * NULL) the final states; initial_state is by sequence; dinitial_state may be NULL.
 * Supported: dk, dv multiples of 16 up to 128; n up to 2^30 (0: the final state is the initial one); B, H up to 65535.
 * Arithmetic: states and every sum in float32.  For bf16 tensors the weighted products of a chunk's rows (64 of them) and the
 * state as an operand of an output are rounded to bf16 once, as the output is: 2.3e-3 of an output in the 2-norm, where rounding the
 * output alone leaves 1.7e-3; what goes into a state is not.  wersa_decay_step rounds its output only.  A row that is not finite reaches
 * only what depends on it, which is then not finite, and may be NaN where the definition has an infinity.  The other conventions are those above.
 */
typedef struct {
  int32_t B, H, n, dk, dv;
  int32_t dtype;           /* wersa_dtype of q, k, v, out and their gradients */
  int32_t packed;
  float scale;
  int64_t stride_q[3], stride_k[3], stride_v[3], stride_o[3];
  int64_t stride_dq[3], stride_dk[3], stride_dv[3];   /* of the gradients; three zeros: those of q, k, v */
  int32_t clear;           /* packed: 1: the forward writes zeros to the rows of out that are of no sequence */
} wersa_decay_desc;

size_t wersa_decay_workspace_bytes(const wersa_decay_desc *desc, int for_backward);
size_t wersa_decay_saved_bytes(const wersa_decay_desc *desc);

wersa_status wersa_decay_forward(const wersa_decay_desc *desc, const void *q, const void *k, const void *v,
                                 const float *log_decay, const int32_t *offsets, const float *initial_state,
                                 float *final_state, const int32_t *slots, int32_t state_slots, void *out, void *saved,
                                 void *workspace, size_t workspace_bytes, void *hip_stream);

wersa_status wersa_decay_backward(const wersa_decay_desc *desc, const void *q, const void *k, const void *v,
                                  const float *log_decay, const int32_t *offsets, const float *initial_state,
                                  const void *dout, const float *dfinal_state, const void *saved, void *dq, void *dk,
                                  void *dv, float *dinitial_state, void *workspace, size_t workspace_bytes,
                                  void *hip_stream);

/* One token of each of B sequences (desc->n = 1, not packed): the states are updated in place. */
wersa_status wersa_decay_step(const wersa_decay_desc *desc, const void *q, const void *k, const void *v,
                              const float *log_decay, float *state, const int32_t *slots, int32_t state_slots, void *out,
                              void *hip_stream);

/*
 * Gated linear recurrence, channel by channel (the causal operator whose decay the data choose, for decoders):
 *   a_t = sigmoid(gate_t),  h_t = a_t h_{t-1} + (1 - a_t) x_t,  out_t = h_t
 * over a whole sequence (wersa_recurrence_forward), its derivative (wersa_recurrence_backward), and one token at a time on a cache of states
 * (wersa_recurrence_step).  x, gate and out are (B, n, C), each at strides of its own (batch, row; in elements; channels contiguous); dout is laid out by
 * stride_o.  Any element-aligned pointer is taken.  What is only read may overlap or repeat itself (strides from 0 up); in out, dx and dgate rows and batch entries
 * do not share memory.
 *   packed   0: B sequences of n rows each; offsets is NULL.
 *            1: B sequences of any lengths (zero among them) one behind the other in tensors with one batch entry of n rows, as for decay attention: sequence b
 *               is rows offsets[b] .. offsets[b + 1] - 1; rows of no sequence are left in out as they are, or zeros with clear = 1, and zeros in dx and dgate.
 *   states   float32 [state_slots][C], contiguous: initial_state, final_state and slots as for decay attention (slots in the forward and the step).
 *   saved    what the forward leaves for the backward (wersa_recurrence_saved_bytes, 256-byte aligned); NULL: no backward follows.
 *   workspace  scratch (256-byte aligned) in which workgroups pass states on: of one call at a time.
 * wersa_recurrence_backward: the gradients given those with respect to out and (dfinal_state, by sequence, may be NULL) the final states; initial_state is by
 * sequence; dinitial_state may be NULL, and is none of the buffers that are read.
 * out, dx and dgate are none of the tensors that are read.
 * Supported: n up to 2^30 (0: the final state is the initial one), B up to 65535, C up to 2^20, B n C below 2^43.
 * Arithmetic: states, gates and every sum in float32; what is written is rounded once.  A row that is not finite reaches only what depends on it, which is then not finite.
 * The same bits every time.
 */
typedef struct {
  int32_t B, n, C;
  int32_t dtype;           /* wersa_dtype of x, gate, out and their gradients */
  int32_t packed, clear;
  int64_t stride_x[2], stride_gate[2], stride_o[2];
  int64_t stride_dx[2], stride_dgate[2];   /* read by the backward alone */
} wersa_recurrence_desc;

size_t wersa_recurrence_workspace_bytes(const wersa_recurrence_desc *desc);
size_t wersa_recurrence_saved_bytes(const wersa_recurrence_desc *desc);

wersa_status wersa_recurrence_forward(const wersa_recurrence_desc *desc, const void *x, const void *gate, const int32_t *offsets,
                                      const float *initial_state, float *final_state, const int32_t *slots, int32_t state_slots,
                                      void *out, void *saved, void *workspace, size_t workspace_bytes, void *hip_stream);

wersa_status wersa_recurrence_backward(const wersa_recurrence_desc *desc, const void *x, const void *gate, const int32_t *offsets,
                                       const float *initial_state, const void *dout, const float *dfinal_state, const void *saved,
                                       void *dx, void *dgate, float *dinitial_state, void *workspace, size_t workspace_bytes,
                                       void *hip_stream);

/* One token of each of B sequences (desc->n = 1, not packed): the states are updated in place. */
wersa_status wersa_recurrence_step(const wersa_recurrence_desc *desc, const void *x, const void *gate, float *state,
                                   const int32_t *slots, int32_t state_slots, void *out, void *hip_stream);

/*
 * Root-mean-square norm over the columns of a row, with the residual's addition before it:
 *   r = x + residual (kept in the tensors' type; with residual NULL r is x itself and nothing is written),
 *   y = r * rstd * weight,  rstd = 1 / sqrt(mean(r^2) + eps)
 * The norm reads the stream r as it is kept.  x and residual are (rows, cols) at row strides of their own, at
 * least cols, columns contiguous; r, y, dy, dr and dx are dense.  weight is float32 [cols] or NULL (ones); rstd float32 [rows], NULL:
 * not wanted.  wersa_rms_norm_eight_bit writes y in 8 bits (e4m3, largest value 448) and float32 scales [rows]:
 *   scale = max|y| / 448,  y8 = e4m3(y * (448 / max|y|)) to the nearest, ties to even;  a row of zeros has scale 1.  The bits are
 *   right for rows of any size; below max|y| = 448 * 2^-126 = 5e-36 the scale has fewer than 24 bits, down to zero.
 * wersa_rms_norm_backward: r is the forward's stream (x where no residual was added, at stride_x), dr the gradient that
 * reaches r from elsewhere (NULL: none); dx is the gradient of x and of the residual, dweight (float32 [cols], NULL: not
 * wanted) that of the weight, for which the workspace is needed.  Supported: cols up to 8192, rows up to 2^31 (0: nothing is done but
 * dweight = 0).
 */
typedef struct {
  int64_t rows;
  int32_t cols, dtype;
  float eps;
  int64_t stride_x, stride_residual;
} wersa_norm_desc;

wersa_status wersa_rms_norm_forward(const wersa_norm_desc *desc, const void *x, const void *residual, const float *weight,
                                    void *r, void *y, float *rstd, void *hip_stream);
wersa_status wersa_rms_norm_eight_bit(const wersa_norm_desc *desc, const void *x, const void *residual,
                                      const float *weight, void *r, void *y, float *scales, void *hip_stream);
size_t wersa_rms_norm_workspace_bytes(const wersa_norm_desc *desc);
wersa_status wersa_rms_norm_backward(const wersa_norm_desc *desc, const void *r, const float *weight, const float *rstd,
                                     const void *dy, const void *dr, void *dx, float *dweight, void *workspace,
                                     size_t workspace_bytes, void *hip_stream);

/*
 * Layer norm over the columns of a row, with the residual's addition before it (the conventions, types and limits of the RMS norm):
 *   r = x + residual (kept in the tensors' type; with residual NULL r is x itself and nothing is written),
 *   y = (r - m) * rstd * weight + bias,  m = mean(r),  rstd = 1 / sqrt(mean((r - m)^2) + eps)
 * weight and bias are float32 [cols], either may be NULL (ones, zeros); stats is float32 [rows][2], m and rstd of each row, NULL: not wanted.
 * wersa_layer_norm_backward: dx is the gradient of x and of the residual (dr: what reaches r from elsewhere, NULL: nothing); dweight and dbias
 * (float32 [cols]) may each be NULL: not wanted; for either the workspace is needed.
 */
wersa_status wersa_layer_norm_forward(const wersa_norm_desc *desc, const void *x, const void *residual, const float *weight,
                                      const float *bias, void *r, void *y, float *stats, void *hip_stream);
size_t wersa_layer_norm_workspace_bytes(const wersa_norm_desc *desc);
wersa_status wersa_layer_norm_backward(const wersa_norm_desc *desc, const void *r, const float *weight, const float *stats,
                                       const void *dy, const void *dr, void *dx, float *dweight, float *dbias, void *workspace,
                                       size_t workspace_bytes, void *hip_stream);

/*
 * Rows of an embedding for tokens, and the gradient of its weights:
 *   out[i] = scale * weight[token_i],   dweight[v] = scale * (sum of dout[i] over the places i with token_i = v)
 * A token below 0 or from vocabulary on has no row: zeros in out, and no part in dweight (a batch's padding, rows that another device holds).
 * tokens: device integers of token_bytes (4 or 8), contiguous.  weight (vocabulary, cols) at rows of stride_weight, out (tokens, cols) at rows of
 * stride_out, at least cols; wersa_embedding_backward reads dout at stride_out and writes every row of dweight at stride_weight, those of tokens
 * that are nowhere with zeros.  Columns contiguous; any element-aligned pointer is taken (the workspace: 256 bytes).  Types: dtype of out and dout,
 * weight_dtype of weight and dweight.  Sums in float32, places in their order within pieces of the sorted list and these in theirs: the same bits every time.
 * Supported: tokens below 2^31 (0: zeros in dweight), vocabulary below 2^31, cols up to 2^20.
 */
typedef struct {
  int64_t tokens;
  int32_t vocabulary, cols;
  int32_t dtype, weight_dtype; /* wersa_dtype of out and dout, of weight and dweight */
  int32_t token_bytes;
  float scale;
  int64_t stride_weight, stride_out;
} wersa_embedding_desc;

wersa_status wersa_embedding_forward(const wersa_embedding_desc *desc, const void *tokens, const void *weight, void *out,
                                     void *hip_stream);
size_t wersa_embedding_workspace_bytes(const wersa_embedding_desc *desc);
wersa_status wersa_embedding_backward(const wersa_embedding_desc *desc, const void *tokens, const void *dout, void *dweight,
                                      void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Logits before a token is chosen: penalties for tokens that were there before, biases, a mask of bits.  For each of B rows and each token v, in float32 and
 * in this order:
 *   v in the row's history:  z = z > 0 ? z / repetition : z * repetition
 *                            z -= frequency * count + (count > 0 ? presence : 0),  count: how often v is in the history behind the prompt
 *   biases:                  z += the biases of v, in their order
 *   v not allowed:           z = -infinity, whatever it was (a row that allows nothing is all -infinity)
 * logits and out are (B, vocabulary) at row strides of their own, columns contiguous, and may be the same buffer; any element-aligned pointer is taken.
 *   history  int32 [history_rows][history_most] at rows of stride_history, or NULL; lengths int32 [history_rows] (clamped to 0 .. history_most) and
 *            prompt_lengths int32 [history_rows] (NULL: none): how many tokens there are, and how many of the first of them are the
 *            prompt.  slots int32 [B] or NULL: row b has history slots[b], or b; one below 0 or from history_rows on is none.
 *   repetition, presence, frequency  float32 [B], each may be NULL (1, 0, 0).  repetition is above 0.
 *   biases   how many a row has: bias_tokens int32 and bias_values float32 [B][biases] at rows of stride_bias (0: the same for every row).
 *   mask     32-bit words [B][(vocabulary + 31) / 32] at rows of stride_mask (0: the same for every row) or NULL; token v is bit v % 32 of word v / 32,
 *            1: allowed.
 * Tokens outside 0 .. vocabulary - 1 in a history or among the biases are passed over.
 * Supported: B up to 65535, biases up to 1023, history_most below 2^21.
 */
typedef struct {
  int32_t B, vocabulary, dtype; /* wersa_dtype of logits and out */
  int32_t history_rows, history_most, biases;
  int64_t stride_logits, stride_out, stride_history, stride_bias, stride_mask;
} wersa_logits_desc;

wersa_status wersa_logits_adjust(const wersa_logits_desc *desc, const void *logits, const int32_t *history, const int32_t *lengths,
                                 const int32_t *prompt_lengths, const int32_t *slots, const float *repetition,
                                 const float *presence, const float *frequency, const int32_t *bias_tokens,
                                 const float *bias_values, const uint32_t *mask, void *out, void *hip_stream);

/* 1 if this descriptor runs on the MFMA path, 0 if on the generic path, -1 if rejected. */
int32_t wersa_selected_path(const wersa_desc *desc);

/* Offsets (in floats) of the pieces inside `saved`, for tests and tools:
 * which = 0 S [B*H][m][d], 1 z [B*H][m], 2 qbar [B*H][d], 3 gate sigmoid s [B*H][L+1],
 * 4 F [B*H][L+1], 5 D [B*H][n]. Returns -1 on a bad argument. */
int64_t wersa_saved_offset(const wersa_desc *desc, int which);

/*
 * Optional per-kernel timing for benchmarks and tools (off by default; the only mutable
 * library state, not thread-safe). While enabled, each kernel launch is bracketed by a HIP
 * event pair on the caller's stream. wersa_profile_collect waits for the recorded events,
 * sums the elapsed time per kernel name, clears the recording and returns the number of
 * distinct names; wersa_profile_get copies entry `index` (0 on success, 1 on bad argument).
 * wersa_profile_only restricts the bracketing to launches of one kernel name (NULL or "" =
 * every launch), so that timing one kernel does not put event records between all the others.
 */
void wersa_profile_enable(int on);
void wersa_profile_only(const char *name);
void wersa_profile_reset(void);
int32_t wersa_profile_collect(void);
int32_t wersa_profile_get(int32_t index, char *name, int32_t name_len, double *total_ms,
                          int32_t *launches);

/*
 * Reference microbenchmarks for benchmarks and tools: what this device sustains, measured in the
 * calling process, next to the nominal peaks.  Both enqueue on hip_stream, WAIT for the result and
 * return it (-1.0 on a bad argument or a failed launch).
 * wersa_peak_copy: a plain streaming copy of `bytes` (multiple of 16; dst, src device pointers,
 * 16-byte aligned, not overlapping) repeated `reps` times; returns GB/s, read plus written.
 * wersa_peak_mfma: `reps` launches of a loop of independent v_mfma_f32_32x32x16_bf16 on every
 * compute unit, operands in registers; returns TFLOP/s.  `sink` is one float of device memory
 * (never written in practice).
 */
double wersa_peak_copy(void *dst, const void *src, size_t bytes, int32_t reps, void *hip_stream);
double wersa_peak_mfma(float *sink, int32_t reps, void *hip_stream);

const char *wersa_status_string(wersa_status status);

/* Library version, major*10000 + minor*100 + patch.  300: wersa_recurrence_*, wersa_layer_norm_*, wersa_embedding_*, wersa_logits_adjust.  200: wersa_decay_desc has the gradients' strides and clear (a program built
 * against an older header passes a shorter structure, and has to be built again). */
int32_t wersa_version(void);

#ifdef __cplusplus
}
#endif
#endif /* WERSA_H */
