/*
 * hilore.h -- C-ABI of the HiLoRe hot path on AMD Instinct MI355X (gfx950).
 *
 * HiLoRe ("HiLoRe: What to Store, Compress, or Recompute for Efficient GRPO
 * Training") decides, for every saved activation unit of a GRPO actor update,
 * whether to keep it in training precision (H), keep a low-precision copy (L)
 * or recompute it (R).  Per microbatch (Algorithm 1) the data-parallel work is:
 *   after forward   encode the L candidates                 -> hilore_compress
 *   Coefficients    per-token GRPO loss coefficients omega  -> hilore_grpo_coeffs
 *   Exposure, psi   per-unit exposure and risk              -> hilore_unit_exposure_risk
 *   Allocate        joint H/L/R choice under memory and risk -> hilore_allocate
 *   in backward     reconstruct L units                     -> hilore_decompress
 *                   and consume them in the weight gradient -> hilore_dequant_wgrad
 *                   or in the LoRA adapter gradient          -> hilore_dequant_lora_grad
 *                   or in the gated-MLP activation backward  -> hilore_dequant_swiglu_bwd
 * Calibration (App. B.1), before training and between refreshes:
 *   single-unit gradient error y                             -> hilore_grad_rel_err
 *   susceptibility kappa_c and mean reconstruction error     -> hilore_calibrate
 *   psi_u = kappa E_u ebar_u, the risk input of Allocate     -> hilore_risk_score
 * Diagnostics (App. D.3): zero-gradient causes, top-k share  -> hilore_update_sparsity
 * Around them, the layer that recomputes, consumes and trains what the units hold:
 *   norms on leaving a block and entering the next, and back -> hilore_block_norm, hilore_block_norm_bwd
 *   frozen base weights in int8, forward and input gradient  -> hilore_int8_linear, hilore_int8_matmul
 *   optimizer step on the gradients, and their global norm   -> hilore_adamw, hilore_grad_norm
 *   heads of queries and keys: norm and rotation, and back   -> hilore_qk_norm_rope, hilore_qk_norm_rope_bwd
 *   log-probabilities of the chosen tokens, and back         -> hilore_token_logprobs, hilore_token_logprobs_bwd
 *   the loss with its gradient to each log-probability       -> hilore_policy_loss, hilore_preference_loss
 *
 * Conventions shared by every entry point:
 *   - Every tensor pointer is a DEVICE pointer owned by the caller.  The
 *     library never allocates, frees or retains memory, and keeps no state
 *     between calls (the one exception, hilore_unit_exposure_risk_noalloc,
 *     uses a fixed device array of its own).  hilore_unit_desc arrays are
 *     HOST memory, read during the call only.
 *   - `stream` is a hipStream_t passed as void* (NULL = the default stream).
 *     All work is enqueued on it without a host synchronisation; outputs are
 *     valid once the stream reaches them.
 *   - Every argument is validated before anything is launched: on an error
 *     nothing is enqueued and no output is touched.  Validation touches no
 *     device state, so argument errors are reported even without a GPU.
 *   - bf16 tensors are passed as uint16_t* (raw bit patterns).
 *   - Alignment: every tensor pointer must be 16-byte aligned, except the
 *     per-unit outputs of hilore_unit_exposure_risk (4-byte aligned), the
 *     per-unit arrays of hilore_allocate (8-byte aligned for fp64), the
 *     scales of 8-bit optimizer states (4-byte aligned) and, with the alignment
 *     of their elements, positions, inv_freq and all tensors of
 *     hilore_token_logprobs, its backward and the losses (shifted slices of
 *     logits, tokens and masks are theirs).
 *   - The functions are re-entrant; calls on different streams may run
 *     concurrently.  No C++ exception crosses this interface.
 *   - Results do not depend on the launch configuration: every reduction is
 *     done in a fixed order, with no floating-point atomics.
 */
#ifndef HILORE_H
#define HILORE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum hilore_status {
  HILORE_OK = 0,
  HILORE_ERR_INVALID_ARG = 1, /* null pointer, negative size, bad enum value      */
  HILORE_ERR_ALIGNMENT = 2,   /* pointer not 16-byte aligned, or bad row stride    */
  HILORE_ERR_UNSUPPORTED = 3, /* valid but unsupported shape (e.g. G > 64)         */
  HILORE_ERR_WORKSPACE = 4,   /* caller-supplied workspace smaller than required   */
  HILORE_ERR_HIP = 5          /* a HIP launch failed (hipGetLastError)             */
} hilore_status;

typedef enum hilore_code {
  HILORE_CODE_INT8 = 0,            /* two's-complement int8, symmetric range [-127, 127],
                                      one fp32 scale per block                          */
  HILORE_CODE_FP8_E4M3FN = 1,      /* OCP E4M3FN (torch.float8_e4m3fn), max 448,
                                      one fp32 scale per block                          */
  HILORE_CODE_FP8_E4M3FN_CAST = 2  /* the paper's literal codec (App. B.1 Eq.
                                      fp8-roundtrip): a plain E4M3FN cast of each bf16
                                      value, no scales (block must be 0, scales unused).
                                      Identical to torch.float8_e4m3fn: nearest-even,
                                      NOT saturating: |x| > 464, +-inf and NaN give the
                                      NaN code 0x7F | sign; (448, 464] gives +-448.  The
                                      cast back is exact; a NaN code gives bf16 0x7FC0. */
} hilore_code;

/* One recovery unit: one saved bf16 activation tensor that receives a single
 * H/L/R action across all its tokens (Sec. 3.4).  Rows are tokens of the
 * microbatch, columns are features; blocks of `block` consecutive columns of
 * one row share one fp32 scale (no scales with HILORE_CODE_FP8_E4M3FN_CAST).
 *   x          bf16 [rows, cols], row stride ld elements (ld >= cols, ld % 8 == 0)
 *   codes      [rows, cols] dense, one byte per element
 *   scales     fp32 [rows, cols / block] dense
 *   xhat       bf16 [rows, cols] dense: output of hilore_decompress
 *   row_ss_x   fp32 [rows] or NULL: per-row sum of x^2
 *   row_ss_err fp32 [rows] or NULL: per-row sum of (xhat - x)^2
 * Each entry point reads only the fields it names. */
typedef struct hilore_unit_desc {
  const uint16_t *x;
  void *codes;
  float *scales;
  uint16_t *xhat;
  float *row_ss_x;
  float *row_ss_err;
  int64_t rows;
  int64_t cols;
  int64_t ld;
} hilore_unit_desc;

/* Human-readable name of a status code (static storage; never NULL). */
const char *hilore_status_string(int status);

/* Library version as 10000 * major + 100 * minor + patch. */
int hilore_version(void);

/*
 * GRPO update quantities for P prompts x G responses x T token slots
 * (Sec. 3.1 Eq. grpo-objective; Sec. 3.2 Eq. update-coefficient; the K3 KL
 * derivative in the proof of Prop. 1; advantages as in App. D.1.1).
 *
 *   rewards  f32 [P*G]          response rewards, prompt-major (group i = rows iG..iG+G-1)
 *   logp_new f32 [P*G*T]        s_t, current-policy log-prob of each slot (response-major)
 *   logp_old f32 [P*G*T]        s_t^old
 *   logp_ref f32 [P*G*T]        s_t^ref; may be NULL only when beta == 0
 *   mask     u8  [P*G*T]        update mask m_t (nonzero = valid); NULL = all valid
 *   clip_eps                    clipping radius eps (> 0, < 1)
 *   adv_eps                     advantage stabiliser (the paper uses 1e-6)
 *   beta                        K3 KL weight (>= 0)
 *   n_norm                      N, the normaliser: > 0 uses this value (all valid tokens of
 *                               the complete rollout batch); <= 0 uses the number of valid
 *                               slots in this call
 * Outputs (device):
 *   adv      f32 [P*G]          A = (R - mean_group) / (population std_group + adv_eps),
 *                               group sums formed as a pairwise tree over a power-of-two
 *                               padding of the group (so the result is reproducible bit
 *                               for bit)
 *   ratio    f32 [P*G*T] or NULL  r_t = exp(s_t - s_t^old)
 *   flags    u8  [P*G*T]        bit0: m_t and chi_t (policy term active);
 *                               bit1: m_t and A != 0 and not chi_t (clipped)
 *   coeff    f32 [P*G*T]        omega_t = (m_t / N) (-chi_t r_t A - beta expm1(s_ref - s_t));
 *                               0 where m_t = 0 or N = 0
 * chi_t is decided in log-ratio space: delta = s_t - s_t^old (fp32), chi = delta <= log1p(eps)
 * when A >= 0, else delta >= log1p(-eps), both thresholds rounded to fp32.
 * workspace: used only to count N (n_norm <= 0 with a mask) over more than 2^16
 * slots: then device memory of at least hilore_grpo_coeffs_workspace_bytes(P, G, T)
 * bytes (4 bytes per 2^16 slots, at most 1 KB), 16-byte aligned, contents on entry
 * irrelevant, and calls sharing it must not overlap; otherwise it may be NULL (the
 * query returns 0 for at most 2^16 slots).
 * Limits: 1 <= G <= 64, P >= 0, T >= 0, P*G*T < 2^31.
 * Errors: bad eps or beta, NaN n_norm, null pointers -> INVALID_ARG; G > 64 or too
 * many slots -> UNSUPPORTED; workspace too small when it is needed -> WORKSPACE.
 */
size_t hilore_grpo_coeffs_workspace_bytes(int P, int G, int T);
hilore_status hilore_grpo_coeffs(const float *rewards, const float *logp_new,
                                 const float *logp_old, const float *logp_ref,
                                 const uint8_t *mask, int P, int G, int T, float clip_eps,
                                 float adv_eps, float beta, double n_norm, float *adv,
                                 float *ratio, uint8_t *flags, float *coeff, void *workspace,
                                 size_t workspace_bytes, void *stream);

/*
 * Blockwise absmax encode of the L candidates after forward (App. B.1 Eq.
 * fp8-roundtrip, in the scaled reading: one fp32 scale per 1 x block run of a
 * row; App. B.3 "post-forward encoding").  For every block, with Q = 127
 * (int8) or 448 (E4M3FN) and amax = max |x| over the block:
 *   amax < 2^-64  -> scale 0 and all codes 0;
 *   otherwise      s = amax / Q and r = Q / amax (IEEE fp32 quotients),
 *                  code = RNE(x * r) (int8: clamped to [-127,127]; E4M3FN: saturating),
 *                  scale = s.
 * With row_ss_x / row_ss_err non-NULL the same pass also writes, per row, the
 * fp32 sums of x^2 (for the token RMS weights of Eq. activation-token-weights)
 * and of (xhat - x)^2 with xhat = bf16(value(code) * s) (the reconstruction
 * error of Eq. app-calibration-error), accumulated in a fixed order.
 *   units[n_units]  host array; uses x, codes, scales, row_ss_x, row_ss_err, rows, cols, ld
 *   block           32, 64, 128 or 256; every unit needs cols % block == 0
 * With code HILORE_CODE_FP8_E4M3FN_CAST (block = 0) each element is cast on its
 * own, scales are neither read nor written, and xhat in the row sums is the
 * cast back (a NaN code makes its row's ss_err NaN).
 * All units of one call are encoded on `stream`; they may differ in shape.
 * Errors: bad code, or block != 0 with the cast code -> INVALID_ARG; other
 * block sizes, or a unit of more than 2^30 rows or 2^30 columns -> UNSUPPORTED.
 */
hilore_status hilore_compress(const hilore_unit_desc *units, int n_units, int code, int block,
                              void *stream);

/*
 * Reconstruction of L units for backward (App. B.1 Eq. fp8-roundtrip, the cast
 * back to bf16): xhat = bf16_RNE(value(code) * scale), elementwise; with
 * HILORE_CODE_FP8_E4M3FN_CAST xhat = value(code) exactly (NaN codes -> 0x7FC0).
 *   units[n_units]  host array; uses codes, scales (not with the cast code), xhat, rows, cols
 * Errors as for hilore_compress.
 */
hilore_status hilore_decompress(const hilore_unit_desc *units, int n_units, int code,
                                int block, void *stream);

/*
 * Per-unit exposure and risk for one microbatch (App. B.1 Eqs.
 * activation-token-weights, mlp-weighted-exposure, app-calibration-error;
 * Sec. 3.4 Eq. token-weighted-risk).  T = rows with a nonzero mask byte.
 *   coeff    f32 [rows]  omega_t aligned to activation rows (zero on prompt/padding rows)
 *   mask     u8  [rows]  valid response tokens T; NULL = all rows
 *   units[n_units]       host array; uses row_ss_x, row_ss_err, rows (== rows), cols
 * For each unit u, with a_t = sqrt(ss_x_t / cols):
 *   exposure[u] = sum_{t in T} |omega_t| (a_t + eps_alpha) / (mean_{s in T} a_s + eps_alpha)
 *   risk[u]     = sum_{t in T} |omega_t| sqrt(ss_err_t)
 *   rel_err[u]  = sqrt(sum_t ss_err_t) / (sqrt(sum_t ss_x_t) + eps_rel)   (all rows)
 * exposure and risk are 0 when T is empty.  Outputs are device f32 [n_units].
 * The sums are fp32: partial sums over chunks of 2048 rows of each unit go to
 * `workspace` and are then added in a fixed order (no floating-point atomics,
 * so repeated calls give identical bits).
 * workspace: device memory of at least hilore_unit_exposure_risk_workspace_bytes(rows,
 * n_units) bytes (32 bytes per unit per 2048 rows; 0, and then NULL is allowed, when
 * rows == 0), 16-byte aligned, contents on entry irrelevant; calls sharing it must
 * not overlap.
 * The calibrated risk of App. B.1 Eq. app-risk-score is kappa * exposure * mean rel_err
 * and the additive distortion of Eq. app-distortion sums it over L units; both are
 * host-side scalar steps.
 * Limits: rows < 2^24 (else UNSUPPORTED).  Errors: negative sizes or eps, null
 * pointers, a unit whose rows differ from `rows` -> INVALID_ARG; workspace too
 * small -> WORKSPACE.
 */
size_t hilore_unit_exposure_risk_workspace_bytes(int64_t rows, int n_units);
hilore_status hilore_unit_exposure_risk(const float *coeff, const uint8_t *mask, int64_t rows,
                                        const hilore_unit_desc *units, int n_units,
                                        float eps_alpha, float eps_rel, float *exposure,
                                        float *risk, float *rel_err, void *workspace,
                                        size_t workspace_bytes, void *stream);

/*
 * hilore_unit_exposure_risk without a workspace, for callers that cannot
 * allocate device memory or pass a buffer for it: code under HIP graph
 * capture, tight serving loops, harnesses that forbid allocation.  Same
 * arguments (less the workspace), kernels and results, bit for bit.  The
 * partial sums live in a fixed 1 MiB array in device memory that the library
 * holds on every GPU it runs on until the process ends (its address is looked
 * up once per device, on the first call made with that device current); the
 * call allocates nothing.  One call needs 32 bytes per unit per 2048 rows, so
 * units * ceil(rows / 2048) may be at most 32768 (78 units of 16384 rows use
 * 624), else the call returns WORKSPACE and enqueues nothing.  Every call on
 * one GPU shares that array: calls that overlap on one GPU (other streams,
 * other threads) race and give wrong results; calls in stream order do not.
 * Nothing in the array needs to start at zero.
 */
hilore_status hilore_unit_exposure_risk_noalloc(const float *coeff, const uint8_t *mask,
                                                int64_t rows, const hilore_unit_desc *units,
                                                int n_units, float eps_alpha, float eps_rel,
                                                float *exposure, float *risk, float *rel_err,
                                                void *stream);

/*
 * Weight gradient of a linear layer whose saved input is an L unit, with the
 * reconstruction fused into the GEMM's tile load (the full-parameter setting
 * of App. D "full-parameter" experiments; accumulated over microbatches as in
 * App. D.1.1):
 *   dW[i][j] (+)= sum_t xhat[t][i] * dY[t][j],  xhat = bf16_RNE(value(code[t][i]) * scale[t][i/block])
 *   x_codes  [K, M] one byte per element; x_scales f32 [K, M / block]
 *   dy       bf16 [K, N]; dw f32 [M, N] row-major (the transpose of a [N, M] weight's layout)
 *   accumulate: 0 overwrites dw, 1 adds to it
 * bf16 x bf16 products, fp32 accumulation (MFMA).  xhat is never written to memory.
 * With HILORE_CODE_FP8_E4M3FN_CAST (block = 0, x_scales unused, may be NULL)
 * xhat = value(code) exactly; a NaN code makes its row of dW NaN.
 * Limits: M % block == 0, M % 8 == 0, N % 8 == 0, M and N below 2^22 (else
 * UNSUPPORTED), K >= 0 (K = 0 writes zeros or leaves dw).
 */
hilore_status hilore_dequant_wgrad(const void *x_codes, const float *x_scales, int code,
                                   int block, const uint16_t *dy, float *dw, int64_t K,
                                   int64_t M, int64_t N, int accumulate, void *stream);

/*
 * hilore_dequant_wgrad with a workspace: where the 256x256 tiles of dW do not
 * fill whole rounds of the chip's 256 CUs, the tiles of the last round are
 * split over the tokens, their fp32 partial sums go to `workspace` and are
 * added in ascending token order (no floating-point atomics; the split depends
 * on K, M and N alone, so repeated calls give identical bits; against
 * hilore_dequant_wgrad the rounding of those tiles' sums differs).  Same
 * arguments otherwise, same limits and errors.
 * workspace: device memory of at least hilore_wgrad_workspace_bytes(K, M, N) bytes
 * (at most 128 MB; 0, and then NULL is allowed, where nothing is split), 16-byte
 * aligned, contents on entry irrelevant; calls sharing it must not overlap.  Too
 * small -> WORKSPACE.
 */
size_t hilore_wgrad_workspace_bytes(int64_t K, int64_t M, int64_t N);
hilore_status hilore_dequant_wgrad_ws(const void *x_codes, const float *x_scales, int code,
                                      int block, const uint16_t *dy, float *dw, int64_t K,
                                      int64_t M, int64_t N, int accumulate, void *workspace,
                                      size_t workspace_bytes, void *stream);

/*
 * Gradient of the LoRA down-projection A of a linear layer whose saved input X
 * is an L unit, with the reconstruction fused into the operand load (the
 * paper's default training setting: rank-16 adapters, alpha = 32, on q/k/v/o
 * and gate/up/down, only adapters trainable, App. D.1.1).  With the layer
 * output y = X W^T + scale * (X A^T) B^T and an upstream gradient G, and
 * dh = G B (the gradient of h = X A^T before the scaling):
 *   dA[j][i] (+)= scale * sum_t dh[t][j] * xhat[t][i],
 *   xhat = bf16_RNE(value(code[t][i]) * scale[t][i/block])   (the hilore_decompress value)
 *   x_codes  [K, M] one byte per element; x_scales f32 [K, M / block]
 *   dh       bf16 [K, r] row-major; da f32 [r, M] row-major (the layout of A's gradient)
 *   scale    the adapter scaling alpha / r (applied to the fp32 sum; exact for powers of 2)
 *   accumulate: 0 overwrites da, 1 adds to it
 * bf16 x bf16 products, fp32 accumulation (MFMA), xhat never written to memory;
 * each code is read once per pass of up to 80 adapter rows, so adapters that
 * share one input (q/k/v, gate/up) are best passed side by side in dh (r = 48,
 * 80).  Partial sums over token ranges go to `workspace` and are added in a
 * fixed order (no floating-point atomics).
 * workspace: device memory of at least hilore_lora_grad_workspace_bytes(K, M, r)
 * bytes (below M = 65536 columns: 8 MB per 16 adapter rows of the widest
 * pass, so at most 40 MB), 16-byte aligned, contents on entry irrelevant;
 * calls sharing it must not overlap.
 * With HILORE_CODE_FP8_E4M3FN_CAST (block = 0, x_scales unused) xhat = value(code).
 * Limits: M % block == 0, M % 16 == 0, M < 2^26, K < 2^31, r even, 2 <= r <= 4096.
 * Errors: negative sizes, r < 1, non-finite scale, null pointers -> INVALID_ARG;
 * other shapes (odd r included) -> UNSUPPORTED; workspace too small -> WORKSPACE.
 */
size_t hilore_lora_grad_workspace_bytes(int64_t K, int64_t M, int r);
hilore_status hilore_dequant_lora_grad(const void *x_codes, const float *x_scales, int code,
                                       int block, const uint16_t *dh, float *da, int64_t K,
                                       int64_t M, int r, float scale, int accumulate,
                                       void *workspace, size_t workspace_bytes, void *stream);

/*
 * Joint H/L/R recovery allocation of one microbatch (Sec. 3.4 Eq.
 * joint-allocation, solved exactly on the conservative grid of App. B.2:
 * Eqs. allocation-grid, allocation-integer-costs, allocation-dp, the tie rules
 * and boundary cases that follow them; available actions of App. B.3 Eq.
 * available-recovery-actions).  Actions: 0 = R (recompute; zero utility,
 * memory and risk), 1 = H (keep; tau_h, dm_h, risk 0), 2 = L (low precision;
 * tau_l, dm_l, risk psi).
 *   q[u]         u8: retained representation of unit u under the plan (0/1/2):
 *                H allows {H, L, R}, L allows {L, R}, anything else only R
 *   verified[u]  u8: bit a set when action a is verified for unit u
 *   tau_h, tau_l, dm_h, dm_l, psi   f64 [n_units]: utilities (Delta tau), memory
 *                costs (Delta m) and the L risk (psi_u, e.g. from
 *                hilore_unit_exposure_risk's exposure times the calibration
 *                factor kappa * ebar of App. B.1 Eq. app-risk-score)
 *   m_res        residual memory budget B - M_peak (>= 0), delta_b risk budget (>= 0)
 *   n_b, n_d     grid intervals N_B, N_delta (1024 in the paper), 1 .. 4096
 * A non-R action is available only if verified, allowed by q, with utility
 * > 0 and finite non-negative costs; L also needs delta_b > 0.  Costs round up
 * to integer grid steps (ceil(cost / (budget / n))); a zero budget keeps one
 * state on its axis and admits only zero costs.  Within a state, actions are
 * tried in the order R, H, L and replace the incumbent only when strictly
 * better; the terminal state is the best value, ties to lower risk cost, then
 * lower memory cost; actions come from backtracking.
 * Outputs (device): action u8 [n_units]; totals f64 [3] = (summed utility,
 * memory, risk of the chosen actions, the latter two summed in unit order);
 * jk i64 [2] = terminal integer memory and risk costs.  All arithmetic is
 * fp64 in the order of a sequential implementation, so results are exact.
 * workspace: device memory of at least hilore_allocate_workspace_bytes(n_units,
 * n_b, n_d) bytes, 16-byte aligned, owned by the caller (about 8.9 MB per
 * table plus 279 KB per unit for a 1025 x 1025 grid); its contents on entry
 * do not matter.  Calls that share a workspace must not overlap.
 * Errors: negative or non-finite budgets, n_b or n_d < 1, null pointers ->
 * INVALID_ARG; n_b or n_d > 4096, n_units > 2^20 -> UNSUPPORTED; workspace too
 * small -> WORKSPACE.
 */
size_t hilore_allocate_workspace_bytes(int n_units, int n_b, int n_d);
hilore_status hilore_allocate(int n_units, const uint8_t *q, const uint8_t *verified,
                              const double *tau_h, const double *tau_l, const double *dm_h,
                              const double *dm_l, const double *psi, double m_res,
                              double delta_b, int n_b, int n_d, uint8_t *action, double *totals,
                              int64_t *jk, void *workspace, size_t workspace_bytes,
                              void *stream);

/*
 * Backward of the gated MLP activation h = silu(g) * u (the MLP of the
 * evaluated Qwen/Llama models, whose gate and up activations are complete MLP
 * tensors eligible for L, App. B.1), with an L operand decoded in registers
 * (App. B.1 Eq. fp8-roundtrip; never written to memory):
 *   du = dh * silu(g),   dg = dh * u * sigmoid(g) * (1 + g * (1 - sigmoid(g)))
 *   gate, up   host descriptors of g and u, [rows, cols] each: an L operand gives
 *              codes (+ scales; not with the cast code) and is decoded to exactly
 *              the bf16 value hilore_decompress writes; otherwise x is read as bf16
 *              (row stride ld).  Either or both may be L (then with the same code
 *              and block); rows and cols must agree.
 *   dh         bf16 [rows, cols] dense; dgate, dup bf16 [rows, cols] dense outputs
 * fp32 arithmetic (sigmoid from the hardware exp2 and reciprocal), each output
 * rounded once to bf16.  Limits: cols % 8 == 0, and cols % block == 0 with an L
 * operand.  Errors: null pointers, mismatched shapes -> INVALID_ARG; bad
 * code/block as for hilore_compress; other shapes -> UNSUPPORTED.
 */
hilore_status hilore_dequant_swiglu_bwd(const hilore_unit_desc *gate, const hilore_unit_desc *up,
                                       int code, int block, const uint16_t *dh, uint16_t *dgate,
                                       uint16_t *dup, void *stream);

/*
 * Relative gradient error of one single-unit L intervention, the calibration
 * target y of App. B.1 Eq. app-calibration-error (Sec. 3.4 Eq.
 * calibration-metrics):
 *   y = sqrt( ||g_l - g_ex||^2 / max(||g_ex||^2, eps_num) )    (the paper: eps_num = 1e-30)
 *   g_l, g_ex  f32 [n]: the trainable-parameter gradients with unit u in L and with
 *              exact recovery, e.g. two outputs of hilore_dequant_wgrad (16-byte aligned)
 *   y          f32 [1] (device, 4-byte aligned; may point into the grad_err array of
 *              hilore_calibrate)
 * The sums are fp64 over the fp32 values, in a fixed order (per-workgroup partial
 * sums in `workspace`, then one fixed tree).  workspace: device memory of at least
 * hilore_grad_rel_err_workspace_bytes(n) bytes (at most 16 KB), 16-byte aligned;
 * its contents on entry do not matter; calls sharing it must not overlap.
 * n = 0 gives y = 0.  Errors: n < 0, eps_num not positive and finite, null
 * pointers -> INVALID_ARG; workspace too small -> WORKSPACE.
 */
size_t hilore_grad_rel_err_workspace_bytes(int64_t n);
hilore_status hilore_grad_rel_err(const float *g_l, const float *g_ex, int64_t n, double eps_num,
                                  float *y, void *workspace, size_t workspace_bytes,
                                  void *stream);

/*
 * Calibration of the L risk (App. B.1 Eqs. app-kappa and app-risk-score; Sec.
 * 3.4 Eq. susceptibility), from n_batches calibration microbatches.  Row b of
 * each [n_batches][n_units] f32 array holds, per unit, the exposure E (from
 * hilore_unit_exposure_risk), the reconstruction error e^L (its rel_err output)
 * and the measured gradient error y (hilore_grad_rel_err).  unit_class i32
 * [n_units] gives the class c(u) (saved-state type and layer); units outside
 * [0, n_classes) take no part in any fit.  Outputs (device):
 *   kappa f64 [n_classes]  kappa_c = max(0, sum x y / sum x^2) over the pairs (u, b)
 *                          of class c, x = E e^L: the least-squares fit of y = kappa x
 *                          over kappa >= 0 (0 when sum x^2 = 0)
 *   ebar  f64 [n_units]    mean over b of e^L (0 when n_batches = 0), summed in
 *                          batch order
 * fp64 arithmetic; kappa's sums run in a fixed order.  Errors: negative sizes,
 * null pointers -> INVALID_ARG; n_units * n_batches >= 2^31 -> UNSUPPORTED.
 */
hilore_status hilore_calibrate(int n_units, int n_batches, int n_classes,
                               const int32_t *unit_class, const float *exposure,
                               const float *rel_err, const float *grad_err, double *kappa,
                               double *ebar, void *stream);

/*
 * Calibrated risk of each unit's L action for the current microbatch (App. B.1
 * Eq. app-risk-score, equal to Sec. 3.4 Eq. token-weighted-risk):
 *   psi[u] = kappa[c(u)] * exposure[u] * ebar[u]   (fp64, multiplied in that order)
 * exposure f32 [n_units] from hilore_unit_exposure_risk; kappa, ebar from
 * hilore_calibrate.  A unit whose class is outside [0, n_classes) has psi = +inf,
 * which makes L unavailable in hilore_allocate (psi is its risk input).
 * Errors: negative sizes, null pointers -> INVALID_ARG.
 */
hilore_status hilore_risk_score(int n_units, const int32_t *unit_class, int n_classes,
                                const double *kappa, const double *ebar, const float *exposure,
                                double *psi, void *stream);

/*
 * Structural sparsity of one batch of update coefficients (the diagnostic
 * statistics of App. D.3), over the n = R*T response slots, padding included.
 *   coeff f32 [R*T], flags u8 [R*T], adv f32 [R]: outputs of hilore_grpo_coeffs;
 *   mask u8 [R*T] or NULL (all valid), as passed to it
 * Outputs (device):
 *   counts i64 [3]  slots whose policy gradient is zero, by exclusive cause:
 *                   [0] padding (mask 0), [1] valid slots of a zero-advantage
 *                   response, [2] valid nonzero-advantage slots on the flat clipped
 *                   branch (flag bit 1); divide by n for the fractions
 *   top_share f64 [1]  share of sum |omega| held by the k = max(1, ceil(top_frac * n))
 *                   largest |omega| (padding counts as 0); 0 when every omega is 0
 * The k-th largest |omega| is found exactly (radix select on the fp32 bit patterns)
 * and ties do not change the result; the sums are fp64 in a fixed order.
 * One workgroup (a diagnostic, not a hot-path step).  Errors: negative sizes,
 * top_frac outside (0, 1], null pointers -> INVALID_ARG; R*T >= 2^31 -> UNSUPPORTED.
 */
hilore_status hilore_update_sparsity(const float *coeff, const uint8_t *flags, const float *adv,
                                     const uint8_t *mask, int R, int T, double top_frac,
                                     int64_t *counts, double *top_share, void *stream);

/* How the gate of hilore_block_norm is broadcast over a [rows, cols] block output. */
typedef enum hilore_gate {
  HILORE_GATE_NONE = 0,
  HILORE_GATE_CHANNEL = 1, /* bf16 [cols]: a learned scale of every channel      */
  HILORE_GATE_TOKEN = 2,   /* bf16 [rows]: one value a token, e.g. of a router   */
  HILORE_GATE_ELEMENT = 3  /* bf16 [rows, cols] dense: one value an element      */
} hilore_gate;

/*
 * Leaving a block and entering the next: the norm of the block's output y, its
 * gate, the residual sum with a scale, and the norm before the next block, in one
 * pass over the rows.  With N(v) = v * rsqrt(mean(v^2) + eps) over a row:
 *   h = bf16_RNE(res + scale * gate * (N(y) * w_post))
 *   n = N(h) * w_pre          of h as it is stored, so that a recompute from a kept
 *                             h gives the same n bit for bit
 *   res      bf16 [rows, cols], row stride ld_res (>= cols, % 8 == 0)
 *   y        bf16 [rows, cols], row stride ld_y; NULL: no block output (the norm
 *            before a model's first block): h = res, and w_post and gate must be NULL
 *   w_post   bf16 [cols]; NULL: y enters without a norm
 *   gate     by gate_kind; NULL with HILORE_GATE_NONE
 *   w_pre    bf16 [cols]; NULL: no norm before a next block (then no n, codes, rstd_pre)
 * Outputs, each but one of h, n and codes may be NULL:
 *   h        bf16 [rows, cols] dense; may be res itself where ld_res == cols
 *   n        bf16 [rows, cols] dense
 *   codes    int8 [rows, cols] dense, with code_scales f32 [rows]: n rounded token by
 *            token as hilore_int8_linear rounds its operand (from the fp32 n, not from
 *            its bf16 value), the operand of hilore_int8_matmul
 *   rstd_post, rstd_pre  f32 [rows]: the rsqrt factors of N(y) and N(h), for backward
 * fp32 arithmetic, row sums in a fixed order.  Limits: cols % 8 == 0 (with codes %
 * 16 == 0), cols <= 16384, rows < 2^31.
 */
typedef struct hilore_block_norm_desc {
  const uint16_t *res;
  const uint16_t *y;
  const uint16_t *w_post;
  const uint16_t *gate;
  const uint16_t *w_pre;
  uint16_t *h;
  uint16_t *n;
  int8_t *codes;
  float *code_scales;
  float *rstd_post;
  float *rstd_pre;
  int64_t rows;
  int64_t cols;
  int64_t ld_res;
  int64_t ld_y;
  float scale;
  float eps;
  int gate_kind;
} hilore_block_norm_desc;
hilore_status hilore_block_norm(const hilore_block_norm_desc *d, void *stream);

/*
 * Backward of hilore_block_norm.  With hh = h * rstd_pre, yh = y * rstd_post, means
 * and sums over a row's columns:
 *   D    = dh + rstd_pre * (dn * w_pre - hh * mean(dn * w_pre * hh))
 *   dres = D,   z = yh * w_post,   dz = scale * gate * D
 *   dy   = rstd_post * (dz * w_post - yh * mean(dz * w_post * yh))   (dz without w_post)
 *   dw_pre = sum_rows dn * hh,   dw_post = sum_rows dz * yh,
 *   dgate  = scale * D * z, summed over what the gate was broadcast over
 *   h, y     the saved tensors as units: codes (+ scales) for an L unit, decoded in
 *            registers to the bf16 value hilore_decompress writes; otherwise x, bf16
 *            with row stride ld.  Either may be L (then with the same code and block).
 *            h is read only with dn; y (rows, cols of all zero: none) only with w_post
 *            or a dgate
 *   dn       bf16 [rows, cols], row stride ld_dn, the gradient of n; NULL: none (then
 *            w_pre, rstd_pre, dw_pre must be NULL)
 *   dh       bf16 [rows, cols] dense, the gradient that reaches h past the next block;
 *            NULL: none
 * Outputs, each may be NULL (frozen weights take no dw_*, no dgate of a channel):
 *   dres, dy bf16 [rows, cols] dense; dres may be dh itself
 *   dw_pre, dw_post f32 [cols]; dgate f32 [cols], f32 [rows] or bf16 [rows, cols] by
 *   gate_kind.  accumulate != 0 adds dw_pre, dw_post and a channel's dgate to what is
 *   there; all other outputs are overwritten.
 * fp32 arithmetic; the sums over rows go to `workspace` by workgroups and are added in
 * a fixed order (no floating-point atomics).  workspace: device memory of at least
 * hilore_block_norm_bwd_workspace_bytes(d) bytes (0, and then NULL is allowed, without
 * sums over rows), 16-byte aligned, contents on entry irrelevant; calls sharing it must
 * not overlap.  Limits as for hilore_block_norm; with L units cols % block == 0.
 */
typedef struct hilore_block_norm_bwd_desc {
  hilore_unit_desc h;
  hilore_unit_desc y;
  const uint16_t *w_post;
  const uint16_t *gate;
  const uint16_t *w_pre;
  const float *rstd_post;
  const float *rstd_pre;
  const uint16_t *dn;
  const uint16_t *dh;
  uint16_t *dres;
  uint16_t *dy;
  float *dw_post;
  float *dw_pre;
  void *dgate;
  int64_t rows;
  int64_t cols;
  int64_t ld_dn;
  float scale;
  int gate_kind;
} hilore_block_norm_bwd_desc;
size_t hilore_block_norm_bwd_workspace_bytes(const hilore_block_norm_bwd_desc *d);
hilore_status hilore_block_norm_bwd(const hilore_block_norm_bwd_desc *d, int code, int block,
                                    int accumulate, void *workspace, size_t workspace_bytes,
                                    void *stream);

/*
 * Linear layer with int8 weights of one scale per output channel (the frozen base
 * weights of the adapter setting, App. D.1.1), its operand rounded to int8 with one
 * scale per token:
 *   a[t][k] = RNE(x'[t][k] * (127 / amax_t)) clamped to [-127, 127],  sa_t = amax_t / 127,
 *             x' = x * factor (fp32), amax_t = max_k |x'[t][k]|  (IEEE fp32 quotients;
 *             amax_t < 2^-64: codes and sa_t are 0; not finite: codes 0, sa_t NaN;
 *             127 times a reciprocal instead of the quotient moves about one code in a million)
 *   out[t][n] (+)= (sum_k a[t][k] * w[n][k]) * sa_t * sw_n + bias[n]
 * The sums are exact in int32 (k <= 131072); the rest is fp32 in that order, rounded
 * once to the output's type.
 *   x        bf16 [tokens, k], row stride ldx (>= k, % 8 == 0); factor f32 [k] or NULL
 *   a        int8 [tokens, k] dense with a_scales f32 [tokens]: codes in hand, for
 *            hilore_int8_matmul (x, ldx and factor are not read)
 *   w        int8 [n, k] dense, values in [-127, 127]; w_scales f32 [n], or NULL: 1
 *   bias     bf16 [n] or NULL
 *   out      bf16 or (out_f32 != 0) f32 [tokens, n], row stride ldo (>= n, % 8 == 0);
 *            accumulate != 0 adds to it (in fp32, rounded once)
 * Gradient of the layer's input, dX = (dY * sw) W: hilore_int8_linear with x = dY,
 * factor = w_scales of the layer, w = the layer's codes transposed (once) to [k, n],
 * and no w_scales.  Several layers on one input add up with accumulate.
 * hilore_quantize_tokens is the rounding alone; with a weight [n, k] as x it makes
 * the weight's codes and channel scales.
 * workspace: device memory of at least hilore_int8_workspace_bytes(d, quantize) bytes
 * (quantize: 1 for hilore_int8_linear, 0 for hilore_int8_matmul; 0 bytes, and then NULL
 * is allowed, where none is needed), 16-byte aligned, contents on entry irrelevant;
 * calls sharing it must not overlap.
 * Limits: k % 16 == 0, n % 8 == 0, k <= 131072, n < 2^26, tokens < 2^31, tokens * n <=
 * 2^40 (else UNSUPPORTED); k = 0 writes bias or zeros.
 */
typedef struct hilore_int8_desc {
  const uint16_t *x;
  const float *factor;
  const int8_t *a;
  const float *a_scales;
  const int8_t *w;
  const float *w_scales;
  const uint16_t *bias;
  void *out;
  int64_t tokens;
  int64_t k;
  int64_t n;
  int64_t ldx;
  int64_t ldo;
  int out_f32;
  int accumulate;
} hilore_int8_desc;
size_t hilore_int8_workspace_bytes(const hilore_int8_desc *d, int quantize);
hilore_status hilore_int8_linear(const hilore_int8_desc *d, void *workspace,
                                 size_t workspace_bytes, void *stream);
hilore_status hilore_int8_matmul(const hilore_int8_desc *d, void *workspace,
                                 size_t workspace_bytes, void *stream);
hilore_status hilore_quantize_tokens(const uint16_t *x, const float *factor, int64_t tokens,
                                     int64_t k, int64_t ldx, int8_t *codes, float *scales,
                                     void *stream);

/*
 * One tensor of an optimizer step, its gradient and its states.
 *   p        f32 [n] parameters, or NULL; p16 bf16 [n] or NULL.  Both: p is the
 *            parameter and p16 receives its nearest bf16.  p16 alone: the parameter is
 *            bf16 and the new value is rounded up or down at random (below), so that
 *            steps smaller than half a bf16 spacing are not lost
 *   grad     f32 [n], or bf16 [n] with grad_bf16 != 0
 *   m, v     states in 32 bits (m_scales and v_scales NULL): f32 [n], the running means
 *            of g and g^2.  In 8 bits: E4M3FN codes [n] with f32 [ceil(n / 256)] scales
 *            of m and of r = sqrt(v), value = value(code) * scale (scales 4-byte aligned:
 *            those of many tensors may lie one after another)
 *   lr, weight_decay  of this tensor (its parameter group)
 */
typedef struct hilore_adamw_tensor {
  float *p;
  uint16_t *p16;
  const void *grad;
  void *m;
  void *v;
  float *m_scales;
  float *v_scales;
  int64_t n;
  float lr;
  float weight_decay;
  int grad_bf16;
} hilore_adamw_tensor;

/*
 * Global norm of the gradients of many tensors and the factor that clips it:
 *   norm[0] = sqrt(sum over all tensors of g^2),
 *   norm[1] = min(1, max_norm / (norm[0] + 1e-6)), or 1 where max_norm is infinite;
 *             NaN where norm[0] is not finite (hilore_adamw then leaves everything as it is)
 * tensors[n_tensors] is a host array, read during the call; uses grad, grad_bf16, n.
 * norm f32 [2] on the device, 4-byte aligned.  fp64 sums in a fixed order, rounded to
 * fp32's 24 bits; root, sum and quotient are IEEE fp32 operations on that.
 * workspace: device memory of at least hilore_grad_norm_workspace_bytes(tensors,
 * n_tensors) bytes, 16-byte aligned, contents on entry irrelevant; calls sharing it
 * must not overlap.  Errors: max_norm not positive, null pointers, negative sizes ->
 * INVALID_ARG; over 2^40 elements in all -> UNSUPPORTED; workspace too small -> WORKSPACE.
 */
size_t hilore_grad_norm_workspace_bytes(const hilore_adamw_tensor *tensors, int n_tensors);
hilore_status hilore_grad_norm(const hilore_adamw_tensor *tensors, int n_tensors, double max_norm,
                               float *norm, void *workspace, size_t workspace_bytes,
                               void *stream);

/*
 * One AdamW step (decoupled weight decay) over many tensors, g = grad * norm[1]:
 *   m = beta1 m + (1 - beta1) g,   v = beta2 v + (1 - beta2) g^2
 *   p = p (1 - lr weight_decay) - lr (m / (1 - beta1^step)) / (sqrt(v / (1 - beta2^step)) + eps)
 * fp32 arithmetic; the update uses the new states before their rounding, and its quotient is a
 * product with a reciprocal within one unit in the last place.
 *   norm     f32 [2] of hilore_grad_norm, or NULL: g = grad.  Where norm[1] is NaN
 *            nothing is written (a step with an infinite or NaN gradient is skipped)
 *   step     1 for the first step
 *   seed     of the random rounding; give each step its own
 * 8-bit states: per 256 elements scale = amax * (1/448) (0 where amax < 2^-64, as the
 * codec's), codes of |value| * (448 * (1/amax)), and a value between two codes takes the upper one with the probability of
 * its place between them, so that the rounding is unbiased and changes far below a
 * code's spacing, as (1 - beta2) makes them, add up over steps instead of vanishing.
 * r > 0 never becomes code 0: a lost second moment would leave eps alone under m.  A gradient
 * or state that is not finite (in a step that no norm skips) makes its own block so, and no other.
 * Random bits: 32 per element, R = mix(i ^ K), K = mix(seed + 0x9E3779B1 (tensor + 1) + salt)
 * in 32-bit arithmetic with i the element's index (below 2^32) in tensor `tensor` of the
 * call, mix(x): x ^= x >> 16, x *= 0x6A09E667, x ^= x >> 15, x *= 0xBB67AE85, x ^= x >> 16.
 * Salt 0: low half for m, high half for r, as the 16 bits below the code; salt
 * 0x3C6EF372: low half as the 16 bits below a bf16 parameter.  The same inputs and seed
 * give the same bits in every call.
 * All tensors may differ in every field; a launch takes 67 to 100 of them (fewer pointers
 * that any of them has, more tensors).
 * Limits: n < 2^32 for a tensor, addresses below 2^48 (else UNSUPPORTED).  Errors: betas outside [0, 1), eps not
 * a positive normal float, step < 1, null pointers, negative sizes, lr or weight_decay not
 * finite, one of m_scales and v_scales alone -> INVALID_ARG.
 */
hilore_status hilore_adamw(const hilore_adamw_tensor *tensors, int n_tensors, double beta1,
                           double beta2, double eps, int64_t step, const float *norm,
                           uint32_t seed, void *stream);

/* Which columns of a head are rotated together. */
typedef enum hilore_rotation {
  HILORE_ROTATE_HALVES = 0, /* column i with column i + rotated / 2 */
  HILORE_ROTATE_PAIRS = 1   /* column 2i with column 2i + 1         */
} hilore_rotation;

/*
 * From the projections to attention: the norm of every head of the queries and keys
 * and the rotation by its token's position, in one pass.  For head j of token t, x its
 * `dim` columns:
 *   n = x * rsqrt(mean(x^2) + eps) * w      (n = x without w)
 *   (a, b) -> rope_scale * (a cos - b sin, b cos + a sin)  for the i-th two of the first
 *   `rotated` columns of n (rotation), angle = position * inv_freq[i]; other columns of n
 *   as they are
 *   q, k       bf16 [tokens, heads * dim], row strides ld_q and ld_k (a slice of the joint
 *              projection's rows); heads_k may be 0 (k fields unused)
 *   w_q, w_k   bf16 [dim]; NULL: no norm of the queries' / keys' heads
 *   positions  i64 [tokens]; NULL: t.  A negative position is padding: the token's inputs
 *              are not used (they may be NaN) and its outputs are 0
 *   inv_freq   f32 [rotated / 2]; not read where rotated is 0
 * Outputs: q_out, k_out bf16, column c of head j of token t at t * token_stride +
 * j * head_stride + c: [tokens, heads, dim] or [heads, tokens, dim], dense or padded.
 * q_out may be q where the strides are those of q's rows, k_out k likewise.
 * fp32 arithmetic with one rounding at the end; angles in pairs of fp64 (whole turns are taken
 * off before position * inv_freq is rounded: positions up to 2^53 turn as exactly as near ones).
 * Limits: dim % 16 == 0, dim <= 512, rotated % 16 == 0, rotated <= dim, strides % 8 == 0,
 * heads_q + heads_k <= 65536, tokens < 2^31.
 */
typedef struct hilore_qk_norm_rope_desc {
  const uint16_t *q;
  const uint16_t *k;
  const uint16_t *w_q;
  const uint16_t *w_k;
  const int64_t *positions;
  const float *inv_freq;
  uint16_t *q_out;
  uint16_t *k_out;
  int64_t tokens;
  int64_t ld_q;
  int64_t ld_k;
  int64_t q_token_stride;
  int64_t q_head_stride;
  int64_t k_token_stride;
  int64_t k_head_stride;
  int heads_q;
  int heads_k;
  int dim;
  int rotated;
  float eps;
  float rope_scale;
  int rotation;
} hilore_qk_norm_rope_desc;
hilore_status hilore_qk_norm_rope(const hilore_qk_norm_rope_desc *d, void *stream);

/*
 * Backward of hilore_qk_norm_rope.  With g the gradient of a head's output, r its
 * rsqrt factor (formed again from x), means and sums over a head's columns:
 *   dn = g turned back (by -angle) and times rope_scale,   t = dn * w
 *   dx = r * (t - x r * mean(t x r))   (dn without w),   dw = sum over tokens and heads of dn x r
 *   q, k       the saved inputs as units [tokens, heads * dim]: codes (+ scales) for an L
 *              unit, decoded in registers to the bf16 value hilore_decompress writes,
 *              otherwise x, bf16 with row stride ld.  Read only with w_q / w_k; either may
 *              be L (then with the same code and block, heads * dim % block == 0)
 *   dq, dk     bf16, addressed like the forward's outputs; strides may be 0 (one gradient
 *              for all tokens or heads)
 * Outputs: dq_in, dk_in bf16 [tokens, heads * dim], row strides ld_dq and ld_dk (a slice of
 * the projection's gradient); dq_in may be dq where the strides agree; NULL: not wanted.
 * dw_q, dw_k f32 [dim] or NULL; accumulate != 0 adds to what is there.  They may be one tensor (one
 * weight for queries and keys), which gets the sum of both.
 * Tokens with a negative position get 0 and give dw nothing, whatever their rows hold.
 * workspace: device memory of at least hilore_qk_norm_rope_bwd_workspace_bytes(d) bytes (0, and
 * then NULL is allowed, without dw), 16-byte aligned, contents on entry irrelevant; calls
 * sharing it must not overlap.  Sums over tokens and heads in a fixed order.
 */
typedef struct hilore_qk_norm_rope_bwd_desc {
  hilore_unit_desc q;
  hilore_unit_desc k;
  const uint16_t *w_q;
  const uint16_t *w_k;
  const int64_t *positions;
  const float *inv_freq;
  const uint16_t *dq;
  const uint16_t *dk;
  uint16_t *dq_in;
  uint16_t *dk_in;
  float *dw_q;
  float *dw_k;
  int64_t tokens;
  int64_t q_token_stride;
  int64_t q_head_stride;
  int64_t k_token_stride;
  int64_t k_head_stride;
  int64_t ld_dq;
  int64_t ld_dk;
  int heads_q;
  int heads_k;
  int dim;
  int rotated;
  float eps;
  float rope_scale;
  int rotation;
} hilore_qk_norm_rope_bwd_desc;
size_t hilore_qk_norm_rope_bwd_workspace_bytes(const hilore_qk_norm_rope_bwd_desc *d);
hilore_status hilore_qk_norm_rope_bwd(const hilore_qk_norm_rope_bwd_desc *d, int code, int block,
                                      int accumulate, void *workspace, size_t workspace_bytes,
                                      void *stream);

/*
 * Log-probabilities of chosen tokens, from logits z (the s_t of the update coefficient,
 * Sec. 3.2).  For a row with target t, over its `vocab` columns:
 *   m = max z,   S = sum exp(scale (z - m)),   logp = scale (z_t - m) - log S
 *   entropy = log S - sum p scale (z - m),   p = exp(scale (z - m)) / S
 *   logits   bf16 or (logits_f32 != 0) f32 [rows, vocab], row stride ld (>= vocab, any
 *            value: rows may begin anywhere)
 *   targets  i64 [rows].  A negative target is a row without a token: it is not read and
 *            its outputs are 0.  A target >= vocab gives logp NaN
 *   scale    1 / temperature, from 2^-126 to 2^127
 * Outputs f32 [rows], each may be NULL: logp, entropy, row_max = m and log_sum = log S
 * (which the backward takes: m and log S apart keep what their sum would round away).
 * Columns of -inf have p = 0; a row of nothing else, or with +inf or NaN, gives NaN.  Logits
 * further below m than the largest fp32 count as infinitely far, whatever the scale.
 * fp32 arithmetic.  S is summed without the chosen token's own term, which is added last: where
 * it is nearly all of S, logp = -log1p(the rest) keeps its relative precision.  A
 * row's bits do not depend on the other rows of the call.
 * workspace: device memory of at least hilore_token_logprobs_workspace_bytes(d) bytes (few
 * long rows are split over workgroups; 0, and then NULL is allowed, for others), 16-byte aligned,
 * contents on entry irrelevant; calls sharing it must not overlap.
 * Limits: rows < 2^31, vocab < 2^28; vocab = 0 only with rows = 0.
 */
typedef struct hilore_token_logprobs_desc {
  const void *logits;
  const int64_t *targets;
  float *logp;
  float *entropy;
  float *row_max;
  float *log_sum;
  int64_t rows;
  int64_t vocab;
  int64_t ld;
  float scale;
  int logits_f32;
} hilore_token_logprobs_desc;
size_t hilore_token_logprobs_workspace_bytes(const hilore_token_logprobs_desc *d);
hilore_status hilore_token_logprobs(const hilore_token_logprobs_desc *d, void *workspace,
                                    size_t workspace_bytes, void *stream);

/*
 * Backward of hilore_token_logprobs, with l_j = scale (z_j - m) - log S and p_j = exp(l_j):
 *   dz_j = scale (dlogp (1[j = t] - p_j) - dentropy p_j (l_j + entropy))
 *   row_max, log_sum, entropy   as the forward wrote them (entropy only with dentropy)
 *   dlogp f32 [rows], dentropy f32 [rows] or NULL
 *   dlogits  of the logits' type [rows, vocab], row stride ld_out (>= vocab, any value);
 *            may be the logits themselves where the strides agree
 * Rows with a negative target, or with dlogp and dentropy both 0 (padding, clipped tokens
 * and responses without advantage), are not read: their gradient is 0.  A target >= vocab
 * gives a row of NaN.  Limits as for hilore_token_logprobs.
 */
typedef struct hilore_token_logprobs_bwd_desc {
  const void *logits;
  const int64_t *targets;
  const float *row_max;
  const float *log_sum;
  const float *entropy;
  const float *dlogp;
  const float *dentropy;
  void *dlogits;
  int64_t rows;
  int64_t vocab;
  int64_t ld;
  int64_t ld_out;
  float scale;
  int logits_f32;
} hilore_token_logprobs_bwd_desc;
hilore_status hilore_token_logprobs_bwd(const hilore_token_logprobs_bwd_desc *d, void *stream);

typedef enum hilore_ratio {
  HILORE_RATIO_TOKEN = 0,   /* exp(s_t - s_t^old) of each token                         */
  HILORE_RATIO_SEQUENCE = 1 /* exp of the mean of s - s^old over a sequence's valid tokens */
} hilore_ratio;
typedef enum hilore_kl {
  HILORE_KL_NONE = 0,
  HILORE_KL_K1 = 1, /* x = s - s_ref       */
  HILORE_KL_K2 = 2, /* x^2 / 2             */
  HILORE_KL_K3 = 3  /* exp(-x) - 1 + x     */
} hilore_kl;
typedef enum hilore_mean {
  HILORE_MEAN_TOKENS = 0,   /* weight of a valid token: 1 / N                            */
  HILORE_MEAN_SEQUENCES = 1 /* 1 / (N n_i), n_i the valid tokens of its sequence          */
} hilore_mean;

/*
 * Clipped policy loss with a KL term and an entropy bonus (Sec. 3.1 Eq. grpo-objective and
 * its usual variants): its value, its statistics and its gradient to each log-probability
 * and entropy.  For a valid token with advantage A and log ratio delta:
 *   chi    = not (delta > log1p(clip_high) where A >= 0, delta < log1p(-clip_low) where A < 0;
 *            thresholds rounded to fp32, as in hilore_grpo_coeffs) and, with dual_clip > 0
 *            and A < 0, not delta > log(dual_clip); dual_clip is 0 or above 1.  So a NaN stays
 *   policy = -A r where chi holds, r = exp(delta), else -A times the bound that delta is past
 *            (1 + clip_high, 1 - clip_low or dual_clip); 0 where A = 0
 *   loss   = sum over valid tokens of weight * (policy + beta * kl - entropy_weight * entropy)
 *            (a KL or entropy of weight 0 is not in it, be it infinite or NaN, only in its statistic)
 *   dlogp  = weight * (-chi A r + beta * dkl/ds),   dentropy = -entropy_weight * weight
 *            (with HILORE_RATIO_SEQUENCE too: the ratio moves by 1 / n_i with each token, and
 *            the n_i tokens of the sequence share it)
 * Sequences: rows of equal length n_tokens / sequences one after another, or with
 * offsets i64 [sequences + 1] (nondecreasing, within [0, n_tokens]) sequence i is the
 * tokens [offsets[i], offsets[i + 1]), possibly none.  Tokens of no sequence count for
 * nothing and their outputs are left as they were.
 *   logp, logp_old, logp_ref, entropy  f32 [n_tokens]; logp_ref only (and always) with a kl,
 *            entropy NULL: no bonus (entropy_weight 0, dentropy NULL)
 *   adv      f32 [sequences], or (adv_per_token != 0) [n_tokens], then with HILORE_RATIO_TOKEN
 *   mask     u8 [n_tokens] (nonzero = valid), NULL: all.  What is masked is not used, be it
 *            infinite or NaN
 *   n_norm   N: > 0 uses this value (of the complete batch); else the number of valid tokens
 *            (HILORE_MEAN_TOKENS) or of sequences that have any (HILORE_MEAN_SEQUENCES) of
 *            this call.  Without a valid token loss and gradients are 0
 * Outputs, each may be NULL: dlogp, dentropy, token_loss (a token's part of the loss) f32
 * [n_tokens], 0 where masked; flags u8 [n_tokens]: bit 0 valid and chi, bit 1 valid, A != 0
 * and not chi; stats f32 [8]: loss, weighted sums of policy, kl and entropy, share of the
 * valid tokens with flag bit 1, their mean ratio, their number, the sequences that have any.
 * Per-token arithmetic in fp32; statistics are summed in fp32 over at most 256 tokens and in fp64
 * beyond, a sequence's mean in fp64, all in a fixed order.
 * workspace: device memory of at least hilore_policy_loss_workspace_bytes(d) bytes, 16-byte
 * aligned, contents on entry irrelevant; calls sharing it must not overlap.
 * Limits: n_tokens < 2^31, sequences < 2^31.
 */
typedef struct hilore_policy_loss_desc {
  const float *logp;
  const float *logp_old;
  const float *logp_ref;
  const float *entropy;
  const float *adv;
  const uint8_t *mask;
  const int64_t *offsets;
  float *dlogp;
  float *dentropy;
  float *token_loss;
  uint8_t *flags;
  float *stats;
  int64_t n_tokens;
  int64_t sequences;
  double n_norm;
  float clip_low;
  float clip_high;
  float dual_clip;
  float beta;
  float entropy_weight;
  int adv_per_token;
  int ratio;
  int kl;
  int mean;
} hilore_policy_loss_desc;
size_t hilore_policy_loss_workspace_bytes(const hilore_policy_loss_desc *d);
hilore_status hilore_policy_loss(const hilore_policy_loss_desc *d, void *workspace,
                                 size_t workspace_bytes, void *stream);

typedef enum hilore_preference {
  HILORE_PREFERENCE_LOGISTIC = 0, /* (1 - e) softplus(-beta h) + e softplus(beta h), e = label_smoothing */
  HILORE_PREFERENCE_HINGE = 1,    /* max(0, 1 - beta h)      */
  HILORE_PREFERENCE_SQUARED = 2   /* (h - 1 / (2 beta))^2    */
} hilore_preference;

/*
 * Preference loss over pairs of sequences: its value, statistics and its gradient to each
 * log-probability.  With L_i the sum (length_mean != 0: the mean) over the valid tokens of
 * sequence i of logp - logp_ref (logp alone without logp_ref), and h = L_chosen - L_rejected -
 * margin of a pair:
 *   loss = (1 / N) sum over pairs of loss(h);   dlogp of a valid token of sequence i =
 *   (1 / N) (sum of loss'(h) over pairs that choose i - sum over pairs that reject i),
 *   over n_i with length_mean.  An L of -inf (a token that cannot be) gives an infinite h, with
 *   the losses' limits: logistic without smoothing 0 at +inf
 * Sequences, mask and n_tokens as for hilore_policy_loss.
 *   chosen, rejected  i32 [pairs] sequence numbers, or both NULL: pair p is sequences 2p and
 *            2p + 1 (pairs = sequences / 2).  A sequence may be in many pairs, or in none
 *   n_norm   N: > 0 uses this value; else the number of pairs that take part.  A pair takes
 *            no part where a number is negative or one of its sequences has no valid token; a
 *            number >= sequences makes the pair's loss, the statistics and all gradients NaN
 * Outputs, each may be NULL: dlogp f32 [n_tokens], 0 where masked; rewards f32 [sequences] =
 * beta L_i; pair_loss f32 [pairs], 0 for a pair that takes no part; stats f32 [6]: loss, and over the pairs that
 * take part (divided by N) the share with h > 0, the sums of beta h and of the
 * rewards of the chosen and of the rejected, then the number of pairs that take part.
 * Token differences in fp32, sums in fp64 in a fixed order.
 * workspace: device memory of at least hilore_preference_loss_workspace_bytes(d) bytes,
 * 16-byte aligned, contents on entry irrelevant; calls sharing it must not overlap.
 * Limits: n_tokens, sequences, pairs < 2^31; with lists sequences * pairs <= 2^36 (each
 * sequence finds its pairs by reading them).
 */
typedef struct hilore_preference_loss_desc {
  const float *logp;
  const float *logp_ref;
  const uint8_t *mask;
  const int64_t *offsets;
  const int32_t *chosen;
  const int32_t *rejected;
  float *dlogp;
  float *rewards;
  float *pair_loss;
  float *stats;
  int64_t n_tokens;
  int64_t sequences;
  int64_t pairs;
  double n_norm;
  float beta;
  float label_smoothing;
  float margin;
  int loss;
  int length_mean;
} hilore_preference_loss_desc;
size_t hilore_preference_loss_workspace_bytes(const hilore_preference_loss_desc *d);
hilore_status hilore_preference_loss(const hilore_preference_loss_desc *d, void *workspace,
                                     size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* HILORE_H */
