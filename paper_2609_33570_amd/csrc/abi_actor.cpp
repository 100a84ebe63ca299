// C-ABI layer of the operators between an actor's products (heads of queries and keys,
// log-probabilities of chosen tokens, policy and preference loss): argument validation and
// dispatch.  As in abi.cpp every check runs before anything is enqueued and touches no device
// state.
#include "hilore.h"

#include <hip/hip_runtime.h>

#include <cfloat>
#include <cmath>
#include <cstdint>

#include "abi_common.hpp"
#include "hilore_internal.hpp"

namespace {

constexpr int64_t kMaxRows = int64_t(1) << 31;
constexpr int64_t kMaxStride = int64_t(1) << 40;

// Whether every pointer is 16-byte aligned (NULL is).
template <int N>
bool all_aligned16(const void *const (&ptrs)[N]) {
  for (const void *p : ptrs)
    if (!aligned16(p)) return false;
  return true;
}

// Whether every pointer has the alignment of an element of `bytes` (NULL has).
template <int N>
bool all_aligned(uintptr_t bytes, const void *const (&ptrs)[N]) {
  for (const void *p : ptrs)
    if ((reinterpret_cast<uintptr_t>(p) & (bytes - 1)) != 0) return false;
  return true;
}

// ------------------------------------------------------------------ heads --
// What the forward's and the backward's descriptors have in common.
template <class D>
hilore_status check_head_sizes(const D &d) {
  if (d.tokens < 0 || d.heads_q < 0 || d.heads_k < 0 || d.dim < 0 || d.rotated < 0) return HILORE_ERR_INVALID_ARG;
  if (d.rotation != HILORE_ROTATE_HALVES && d.rotation != HILORE_ROTATE_PAIRS) return HILORE_ERR_INVALID_ARG;
  if (!std::isfinite(d.eps) || !(d.eps >= 0.0f) || !std::isfinite(d.rope_scale)) return HILORE_ERR_INVALID_ARG;
  if (d.rotated > d.dim) return HILORE_ERR_INVALID_ARG;
  if (d.dim % 16 != 0 || d.dim > hilore::kHeadMaxDim || d.rotated % 16 != 0 || d.tokens >= kMaxRows ||
      (int64_t)d.heads_q + d.heads_k > 65536)
    return HILORE_ERR_UNSUPPORTED;
  return HILORE_OK;
}

bool fits(int64_t stride) { return stride >= 0 && stride <= kMaxStride; }

// Strides of written heads: token by token or head by head, without overlap.
bool apart(int64_t tokens, int heads, int dim, int64_t token_stride, int64_t head_stride) {
  if (tokens <= 1 && heads <= 1) return true;
  if (heads <= 1) return token_stride >= dim;
  if (tokens <= 1) return head_stride >= dim;
  if (token_stride < dim || head_stride < dim) return false;
  // strides of up to 2^40 times 2^31 tokens: past 64 bits
  const __int128 all_heads = (__int128)(heads - 1) * head_stride + dim;
  const __int128 all_tokens = (__int128)(tokens - 1) * token_stride + dim;
  return token_stride >= all_heads || head_stride >= all_tokens;
}

// Whether heads addressed by both strides lie as in rows `ld` apart.
bool like_rows(int64_t tokens, int heads, int dim, int64_t token_stride, int64_t head_stride, int64_t ld) {
  return (tokens <= 1 || token_stride == ld) && (heads <= 1 || head_stride == dim);
}

hilore_status check_heads_forward(int64_t tokens, int heads, int dim, const uint16_t *x, int64_t ld, const uint16_t *w,
                                  const uint16_t *out, int64_t token_stride, int64_t head_stride) {
  if (heads == 0) return HILORE_OK;
  if (!x || !out || ld < (int64_t)heads * dim || !fits(ld)) return HILORE_ERR_INVALID_ARG;
  if (!fits(token_stride) || !fits(head_stride) || !apart(tokens, heads, dim, token_stride, head_stride))
    return HILORE_ERR_INVALID_ARG;
  if (ld % 8 != 0 || token_stride % 8 != 0 || head_stride % 8 != 0) return HILORE_ERR_ALIGNMENT;
  if (out == x && !like_rows(tokens, heads, dim, token_stride, head_stride, ld)) return HILORE_ERR_INVALID_ARG;
  const void *ptrs[] = {x, w, out};
  return all_aligned16(ptrs) ? HILORE_OK : HILORE_ERR_ALIGNMENT;
}

bool nothing_to_do(int64_t tokens, int heads_q, int heads_k, int dim) {
  return tokens == 0 || heads_q + heads_k == 0 || dim == 0;
}

hilore_status check_heads(const hilore_qk_norm_rope_desc &d) {
  const hilore_status st = check_head_sizes(d);
  if (st != HILORE_OK || nothing_to_do(d.tokens, d.heads_q, d.heads_k, d.dim)) return st;
  const hilore_status q = check_heads_forward(d.tokens, d.heads_q, d.dim, d.q, d.ld_q, d.w_q, d.q_out, d.q_token_stride,
                                              d.q_head_stride);
  if (q != HILORE_OK) return q;
  const hilore_status k = check_heads_forward(d.tokens, d.heads_k, d.dim, d.k, d.ld_k, d.w_k, d.k_out, d.k_token_stride,
                                              d.k_head_stride);
  if (k != HILORE_OK) return k;
  if (d.rotated > 0 && !d.inv_freq) return HILORE_ERR_INVALID_ARG;
  return all_aligned(8, {d.positions}) && all_aligned(4, {d.inv_freq}) ? HILORE_OK : HILORE_ERR_ALIGNMENT;
}

hilore_status check_heads_backward(int64_t tokens, int heads, int dim, const hilore_unit_desc &saved, const uint16_t *w,
                                   const uint16_t *g, int64_t token_stride, int64_t head_stride, const uint16_t *out,
                                   int64_t ld, const float *dw, bool scaled) {
  if (dw && (!w || heads == 0)) return HILORE_ERR_INVALID_ARG;
  if (heads == 0) return HILORE_OK;
  const int64_t cols = (int64_t)heads * dim;
  if (!g || !fits(token_stride) || !fits(head_stride)) return HILORE_ERR_INVALID_ARG;
  if (out && (ld < cols || !fits(ld))) return HILORE_ERR_INVALID_ARG;
  if (token_stride % 8 != 0 || head_stride % 8 != 0 || (out && ld % 8 != 0)) return HILORE_ERR_ALIGNMENT;
  if (out && out == g && !like_rows(tokens, heads, dim, token_stride, head_stride, ld)) return HILORE_ERR_INVALID_ARG;
  if (w) {
    if ((!saved.x && !saved.codes) || saved.rows != tokens || saved.cols != cols) return HILORE_ERR_INVALID_ARG;
    if (saved.codes) {
      if (scaled && !saved.scales) return HILORE_ERR_INVALID_ARG;
      if (!aligned16(saved.codes) || (scaled && !aligned16(saved.scales))) return HILORE_ERR_ALIGNMENT;
    } else {
      if (saved.ld < cols || !fits(saved.ld)) return HILORE_ERR_INVALID_ARG;
      if (saved.ld % 8 != 0 || !aligned16(saved.x)) return HILORE_ERR_ALIGNMENT;
    }
  }
  const void *ptrs[] = {w, g, out, dw};
  return all_aligned16(ptrs) ? HILORE_OK : HILORE_ERR_ALIGNMENT;
}

hilore_status check_heads_bwd(const hilore_qk_norm_rope_bwd_desc &d, int code, int block) {
  const hilore_status st = check_head_sizes(d);
  if (st != HILORE_OK) return st;
  const bool cast = code == HILORE_CODE_FP8_E4M3FN_CAST;
  const bool lq = d.w_q && d.q.codes, lk = d.w_k && d.k.codes;
  if (lq || lk) {
    const hilore_status cb = check_code_block(code, block);
    if (cb != HILORE_OK) return cb;
    if (!cast && ((lq && (int64_t)d.heads_q * d.dim % block != 0) || (lk && (int64_t)d.heads_k * d.dim % block != 0)))
      return HILORE_ERR_UNSUPPORTED;
  }
  if ((d.dw_q && (!d.w_q || d.heads_q == 0)) || (d.dw_k && (!d.w_k || d.heads_k == 0))) return HILORE_ERR_INVALID_ARG;
  if (!aligned16(d.dw_q) || !aligned16(d.dw_k)) return HILORE_ERR_ALIGNMENT;
  if (nothing_to_do(d.tokens, d.heads_q, d.heads_k, d.dim)) return HILORE_OK;
  const hilore_status q = check_heads_backward(d.tokens, d.heads_q, d.dim, d.q, d.w_q, d.dq, d.q_token_stride,
                                               d.q_head_stride, d.dq_in, d.ld_dq, d.dw_q, !cast);
  if (q != HILORE_OK) return q;
  const hilore_status k = check_heads_backward(d.tokens, d.heads_k, d.dim, d.k, d.w_k, d.dk, d.k_token_stride,
                                               d.k_head_stride, d.dk_in, d.ld_dk, d.dw_k, !cast);
  if (k != HILORE_OK) return k;
  if (d.rotated > 0 && !d.inv_freq) return HILORE_ERR_INVALID_ARG;
  return all_aligned(8, {d.positions}) && all_aligned(4, {d.inv_freq}) ? HILORE_OK : HILORE_ERR_ALIGNMENT;
}

template <class D>
hilore::HeadsArgs head_sizes(const D &d) {
  hilore::HeadsArgs a{};
  a.positions = d.positions;
  a.inv_freq = d.inv_freq;
  a.tokens = d.tokens;
  a.heads_q = d.heads_q;
  a.heads_k = d.heads_k;
  a.dim = d.dim;
  a.rotated = d.rotated;
  a.eps = d.eps;
  a.inv_dim = d.dim ? (float)(1.0 / (double)d.dim) : 0.0f;
  a.rope_scale = d.rope_scale;
  a.pairs = d.rotation == HILORE_ROTATE_PAIRS;
  return a;
}

hilore::HeadSide bwd_side(const hilore_unit_desc &saved, const uint16_t *w, const uint16_t *g, uint16_t *out,
                          int64_t token_stride, int64_t head_stride, int64_t ld, float *dw, bool scaled) {
  hilore::HeadSide s{};
  if (w) {  // the saved rows are read only where there is a norm
    s.in.codes = static_cast<const uint8_t *>(saved.codes);
    s.in.x = saved.codes ? nullptr : saved.x;
    s.in.scales = saved.codes && scaled ? saved.scales : nullptr;
    s.in.ld = saved.ld;
  }
  s.w = w;
  s.g = g;
  s.out = out;
  s.token_stride = token_stride;
  s.head_stride = head_stride;
  s.ld_out = ld;
  s.dw = dw;
  return s;
}

// Of the power of two that a block is; 0 for what stands there where no unit has blocks.
int log2_of(int block) {
  int l = 0;
  while (l < 30 && (1 << l) < block) ++l;
  return (1 << l) == block ? l : 0;
}

// --------------------------------------------------------------- logprobs --
// scale log2(e) has to be finite.
hilore_status check_logits(int64_t rows, int64_t vocab, float scale) {
  if (rows < 0 || vocab < 0 || (rows > 0 && vocab == 0)) return HILORE_ERR_INVALID_ARG;
  if (!(scale >= FLT_MIN) || !(scale <= 0x1p127f)) return HILORE_ERR_INVALID_ARG;
  if (rows >= kMaxRows || vocab >= (int64_t(1) << 28)) return HILORE_ERR_UNSUPPORTED;
  return HILORE_OK;
}

hilore_status check_logprobs(const hilore_token_logprobs_desc &d) {
  const hilore_status st = check_logits(d.rows, d.vocab, d.scale);
  if (st != HILORE_OK || d.rows == 0) return st;
  if (!d.logits || !d.targets || d.ld < d.vocab || !fits(d.ld)) return HILORE_ERR_INVALID_ARG;
  return all_aligned(d.logits_f32 ? 4 : 2, {d.logits}) && all_aligned(8, {d.targets}) &&
                 all_aligned(4, {d.logp, d.entropy, d.row_max, d.log_sum})
             ? HILORE_OK
             : HILORE_ERR_ALIGNMENT;
}

hilore_status check_logprobs_bwd(const hilore_token_logprobs_bwd_desc &d) {
  const hilore_status st = check_logits(d.rows, d.vocab, d.scale);
  if (st != HILORE_OK || d.rows == 0) return st;
  if (!d.logits || !d.targets || !d.row_max || !d.log_sum || !d.dlogp || !d.dlogits) return HILORE_ERR_INVALID_ARG;
  if (d.dentropy && !d.entropy) return HILORE_ERR_INVALID_ARG;
  if (d.ld < d.vocab || d.ld_out < d.vocab || !fits(d.ld) || !fits(d.ld_out)) return HILORE_ERR_INVALID_ARG;
  if (d.dlogits == d.logits && d.rows > 1 && d.ld != d.ld_out) return HILORE_ERR_INVALID_ARG;
  return all_aligned(d.logits_f32 ? 4 : 2, {d.logits, d.dlogits}) && all_aligned(8, {d.targets}) &&
                 all_aligned(4, {d.row_max, d.log_sum, d.entropy, d.dlogp, d.dentropy})
             ? HILORE_OK
             : HILORE_ERR_ALIGNMENT;
}

// ----------------------------------------------------------------- losses --
hilore_status check_sequences(int64_t tokens, int64_t sequences, const int64_t *offsets, double n_norm) {
  if (tokens < 0 || sequences < 0 || n_norm != n_norm || std::isinf(n_norm)) return HILORE_ERR_INVALID_ARG;
  if (tokens >= kMaxRows || sequences >= kMaxRows) return HILORE_ERR_UNSUPPORTED;
  if (!offsets && (sequences == 0 ? tokens != 0 : tokens % sequences != 0)) return HILORE_ERR_INVALID_ARG;
  return HILORE_OK;
}

hilore::SequencesArgs sequences_of(const int64_t *offsets, const uint8_t *mask, int64_t tokens, int64_t sequences) {
  hilore::SequencesArgs q{};
  q.offsets = offsets;
  q.mask = mask;
  q.tokens = tokens;
  q.sequences = sequences;
  q.length = sequences ? tokens / sequences : 0;
  return q;
}

hilore_status check_policy(const hilore_policy_loss_desc &d) {
  if (!(d.clip_low > 0.0f) || !(d.clip_low < 1.0f) || !(d.clip_high > 0.0f) || !std::isfinite(d.clip_high) ||
      !std::isfinite(d.dual_clip) || d.dual_clip < 0.0f || !std::isfinite(d.beta) || !std::isfinite(d.entropy_weight))
    return HILORE_ERR_INVALID_ARG;
  // a bound at or below 1 would cut off an unchanged policy
  if (d.dual_clip > 0.0f && !(d.dual_clip > 1.0f)) return HILORE_ERR_INVALID_ARG;
  if (d.ratio != HILORE_RATIO_TOKEN && d.ratio != HILORE_RATIO_SEQUENCE) return HILORE_ERR_INVALID_ARG;
  if (d.kl < HILORE_KL_NONE || d.kl > HILORE_KL_K3) return HILORE_ERR_INVALID_ARG;
  if (d.mean != HILORE_MEAN_TOKENS && d.mean != HILORE_MEAN_SEQUENCES) return HILORE_ERR_INVALID_ARG;
  const hilore_status st = check_sequences(d.n_tokens, d.sequences, d.offsets, d.n_norm);
  if (st != HILORE_OK) return st;
  if (d.adv_per_token && d.ratio == HILORE_RATIO_SEQUENCE) return HILORE_ERR_UNSUPPORTED;
  if (d.n_tokens > 0) {  // tensors without elements may be NULL
    if (!d.logp || !d.logp_old || (!d.adv && (d.adv_per_token || d.sequences > 0))) return HILORE_ERR_INVALID_ARG;
    if ((d.kl != HILORE_KL_NONE) != (d.logp_ref != nullptr)) return HILORE_ERR_INVALID_ARG;
    if (!d.entropy && (d.entropy_weight != 0.0f || d.dentropy)) return HILORE_ERR_INVALID_ARG;
  }
  return all_aligned(8, {d.offsets}) && all_aligned(4, {d.logp, d.logp_old, d.logp_ref, d.entropy, d.adv, d.dlogp,
                                                        d.dentropy, d.token_loss, d.stats})
             ? HILORE_OK
             : HILORE_ERR_ALIGNMENT;
}

hilore_status check_preference(const hilore_preference_loss_desc &d) {
  if (!std::isfinite(d.beta) || !(d.beta > 0.0f) || !std::isfinite(d.margin)) return HILORE_ERR_INVALID_ARG;
  if (d.loss < HILORE_PREFERENCE_LOGISTIC || d.loss > HILORE_PREFERENCE_SQUARED) return HILORE_ERR_INVALID_ARG;
  if (!(d.label_smoothing >= 0.0f) || !(d.label_smoothing <= 0.5f)) return HILORE_ERR_INVALID_ARG;
  if (d.label_smoothing != 0.0f && d.loss != HILORE_PREFERENCE_LOGISTIC) return HILORE_ERR_INVALID_ARG;
  const hilore_status st = check_sequences(d.n_tokens, d.sequences, d.offsets, d.n_norm);
  if (st != HILORE_OK) return st;
  if (d.pairs < 0 || (d.chosen == nullptr) != (d.rejected == nullptr)) return HILORE_ERR_INVALID_ARG;
  if (!d.chosen && d.pairs != d.sequences / 2 && d.pairs != 0) return HILORE_ERR_INVALID_ARG;
  if (d.pairs >= kMaxRows) return HILORE_ERR_UNSUPPORTED;
  if (d.chosen && d.pairs > 0 && d.sequences > (int64_t(1) << 36) / d.pairs) return HILORE_ERR_UNSUPPORTED;
  if (d.n_tokens > 0 && !d.logp) return HILORE_ERR_INVALID_ARG;
  return all_aligned(8, {d.offsets}) &&
                 all_aligned(4, {d.logp, d.logp_ref, d.chosen, d.rejected, d.dlogp, d.rewards, d.pair_loss, d.stats})
             ? HILORE_OK
             : HILORE_ERR_ALIGNMENT;
}

hilore::PolicyArgs policy_args(const hilore_policy_loss_desc &d) {
  hilore::PolicyArgs a{};
  a.seq = sequences_of(d.offsets, d.mask, d.n_tokens, d.sequences);
  a.logp = d.logp;
  a.old = d.logp_old;
  a.ref = d.logp_ref;
  a.entropy = d.entropy;
  a.adv = d.adv;
  a.dlogp = d.dlogp;
  a.dentropy = d.dentropy;
  a.token_loss = d.token_loss;
  a.stats = d.stats;
  a.flags = d.flags;
  a.n_norm = d.n_norm;
  a.bound_high = (float)(1.0 + (double)d.clip_high);
  a.bound_low = (float)(1.0 - (double)d.clip_low);
  a.log_high = (float)std::log1p((double)d.clip_high);
  a.log_low = (float)std::log1p(-(double)d.clip_low);
  a.dual = d.dual_clip;
  a.log_dual = d.dual_clip > 0.0f ? (float)std::log((double)d.dual_clip) : 0.0f;
  a.beta = d.beta;
  a.bonus = d.entropy_weight;
  a.adv_per_token = d.adv_per_token ? 1 : 0;
  a.sequence_ratio = d.ratio == HILORE_RATIO_SEQUENCE;
  a.kl = d.kl;
  a.sequence_mean = d.mean == HILORE_MEAN_SEQUENCES;
  return a;
}

hilore::PreferenceArgs preference_args(const hilore_preference_loss_desc &d) {
  hilore::PreferenceArgs a{};
  a.seq = sequences_of(d.offsets, d.mask, d.n_tokens, d.sequences);
  a.logp = d.logp;
  a.ref = d.logp_ref;
  a.chosen = d.chosen;
  a.rejected = d.rejected;
  a.dlogp = d.dlogp;
  a.rewards = d.rewards;
  a.pair_loss = d.pair_loss;
  a.stats = d.stats;
  a.pairs = d.pairs;
  a.n_norm = d.n_norm;
  a.beta = d.beta;
  a.smoothing = d.label_smoothing;
  a.margin = d.margin;
  a.loss = d.loss;
  a.length_mean = d.length_mean ? 1 : 0;
  return a;
}

hilore_status check_workspace(const void *workspace, size_t bytes, size_t need) {
  if (need > 0 && !workspace) return HILORE_ERR_INVALID_ARG;
  if (workspace && !aligned16(workspace)) return HILORE_ERR_ALIGNMENT;
  return bytes < need ? HILORE_ERR_WORKSPACE : HILORE_OK;
}

}  // namespace

extern "C" {

hilore_status hilore_qk_norm_rope(const hilore_qk_norm_rope_desc *d, void *stream) {
  if (!d) return HILORE_ERR_INVALID_ARG;
  const hilore_status st = check_heads(*d);
  if (st != HILORE_OK || nothing_to_do(d->tokens, d->heads_q, d->heads_k, d->dim)) return st;
  hilore::HeadsArgs a = head_sizes(*d);
  a.q.in.x = d->q;
  a.q.in.ld = d->ld_q;
  a.q.w = d->w_q;
  a.q.out = d->q_out;
  a.q.token_stride = d->q_token_stride;
  a.q.head_stride = d->q_head_stride;
  if (d->heads_k > 0) {
    a.k.in.x = d->k;
    a.k.in.ld = d->ld_k;
    a.k.w = d->w_k;
    a.k.out = d->k_out;
    a.k.token_stride = d->k_token_stride;
    a.k.head_stride = d->k_head_stride;
  }
  return hip_status(hilore::launch_heads(a, static_cast<hipStream_t>(stream)));
}

size_t hilore_qk_norm_rope_bwd_workspace_bytes(const hilore_qk_norm_rope_bwd_desc *d) {
  if (!d || check_head_sizes(*d) != HILORE_OK || (!d->dw_q && !d->dw_k)) return 0;
  return (size_t)2 * (size_t)hilore::heads_bwd_groups(d->tokens, d->heads_q + d->heads_k, d->dim, 1) * (size_t)d->dim *
         sizeof(float);
}

hilore_status hilore_qk_norm_rope_bwd(const hilore_qk_norm_rope_bwd_desc *d, int code, int block, int accumulate,
                                      void *workspace, size_t workspace_bytes, void *stream) {
  if (!d) return HILORE_ERR_INVALID_ARG;
  const hilore_status st = check_heads_bwd(*d, code, block);
  if (st != HILORE_OK || d->dim == 0 || d->heads_q + d->heads_k == 0) return st;
  const hilore_status ws = check_workspace(workspace, workspace_bytes, hilore_qk_norm_rope_bwd_workspace_bytes(d));
  if (ws != HILORE_OK) return ws;
  const bool scaled = code != HILORE_CODE_FP8_E4M3FN_CAST;
  hilore::HeadsArgs a = head_sizes(*d);
  if (d->heads_q > 0)
    a.q = bwd_side(d->q, d->w_q, d->dq, d->dq_in, d->q_token_stride, d->q_head_stride, d->ld_dq, d->dw_q, scaled);
  if (d->heads_k > 0)
    a.k = bwd_side(d->k, d->w_k, d->dk, d->dk_in, d->k_token_stride, d->k_head_stride, d->ld_dk, d->dw_k, scaled);
  a.accumulate = accumulate ? 1 : 0;
  a.code = code;
  a.block_log2 = log2_of(block);
  a.groups = hilore::heads_bwd_groups(d->tokens, d->heads_q + d->heads_k, d->dim, d->dw_q || d->dw_k);
  a.part = static_cast<float *>(workspace);
  return hip_status(hilore::launch_heads_bwd(a, static_cast<hipStream_t>(stream)));
}

size_t hilore_token_logprobs_workspace_bytes(const hilore_token_logprobs_desc *d) {
  if (!d || check_logits(d->rows, d->vocab, d->scale) != HILORE_OK || d->rows == 0) return 0;
  return hilore::logprobs_part_bytes(d->rows, d->vocab, d->logits_f32 ? 1 : 0);
}

hilore_status hilore_token_logprobs(const hilore_token_logprobs_desc *d, void *workspace, size_t workspace_bytes,
                                    void *stream) {
  if (!d) return HILORE_ERR_INVALID_ARG;
  const hilore_status st = check_logprobs(*d);
  if (st != HILORE_OK || d->rows == 0) return st;
  const hilore_status ws = check_workspace(workspace, workspace_bytes, hilore_token_logprobs_workspace_bytes(d));
  if (ws != HILORE_OK) return ws;
  hilore::LogprobsArgs a{};
  a.logits = d->logits;
  a.targets = d->targets;
  a.logp = d->logp;
  a.entropy = d->entropy;
  a.row_max = d->row_max;
  a.log_sum = d->log_sum;
  a.rows = d->rows;
  a.vocab = d->vocab;
  a.ld = d->ld;
  a.scale = d->scale;
  a.f32 = d->logits_f32 ? 1 : 0;
  a.part = static_cast<float *>(workspace);
  return hip_status(hilore::launch_logprobs(a, static_cast<hipStream_t>(stream)));
}

hilore_status hilore_token_logprobs_bwd(const hilore_token_logprobs_bwd_desc *d, void *stream) {
  if (!d) return HILORE_ERR_INVALID_ARG;
  const hilore_status st = check_logprobs_bwd(*d);
  if (st != HILORE_OK || d->rows == 0) return st;
  hilore::LogprobsBwdArgs a{};
  a.logits = d->logits;
  a.targets = d->targets;
  a.row_max = d->row_max;
  a.log_sum = d->log_sum;
  a.entropy = d->entropy;
  a.dlogp = d->dlogp;
  a.dentropy = d->dentropy;
  a.dlogits = d->dlogits;
  a.rows = d->rows;
  a.vocab = d->vocab;
  a.ld = d->ld;
  a.ld_out = d->ld_out;
  a.scale = d->scale;
  a.f32 = d->logits_f32 ? 1 : 0;
  return hip_status(hilore::launch_logprobs_bwd(a, static_cast<hipStream_t>(stream)));
}

size_t hilore_policy_loss_workspace_bytes(const hilore_policy_loss_desc *d) {
  if (!d || check_sequences(d->n_tokens, d->sequences, d->offsets, d->n_norm) != HILORE_OK) return 0;
  hilore::PolicyArgs a = policy_args(*d);
  return hilore::policy_workspace(a, nullptr);
}

hilore_status hilore_policy_loss(const hilore_policy_loss_desc *d, void *workspace, size_t workspace_bytes, void *stream) {
  if (!d) return HILORE_ERR_INVALID_ARG;
  const hilore_status st = check_policy(*d);
  if (st != HILORE_OK) return st;
  const hilore_status ws = check_workspace(workspace, workspace_bytes, hilore_policy_loss_workspace_bytes(d));
  if (ws != HILORE_OK) return ws;
  hilore::PolicyArgs a = policy_args(*d);
  hilore::policy_workspace(a, workspace);
  return hip_status(hilore::launch_policy(a, static_cast<hipStream_t>(stream)));
}

size_t hilore_preference_loss_workspace_bytes(const hilore_preference_loss_desc *d) {
  if (!d || check_sequences(d->n_tokens, d->sequences, d->offsets, d->n_norm) != HILORE_OK) return 0;
  hilore::PreferenceArgs a = preference_args(*d);
  return hilore::preference_workspace(a, nullptr);
}

hilore_status hilore_preference_loss(const hilore_preference_loss_desc *d, void *workspace, size_t workspace_bytes,
                                     void *stream) {
  if (!d) return HILORE_ERR_INVALID_ARG;
  const hilore_status st = check_preference(*d);
  if (st != HILORE_OK) return st;
  const hilore_status ws = check_workspace(workspace, workspace_bytes, hilore_preference_loss_workspace_bytes(d));
  if (ws != HILORE_OK) return ws;
  hilore::PreferenceArgs a = preference_args(*d);
  hilore::preference_workspace(a, workspace);
  return hip_status(hilore::launch_preference(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
