// C-ABI layer of the layer operators (block norms, int8 products, AdamW): argument
// validation and dispatch.  As in abi.cpp every check runs before anything is
// enqueued and touches no device state.
#include "hilore.h"

#include <hip/hip_runtime.h>

#include <cfloat>
#include <cmath>
#include <cstdint>

#include "abi_common.hpp"
#include "hilore_internal.hpp"

namespace {

bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

// Whether every pointer is 16-byte aligned (NULL is).
template <int N>
bool all_aligned16(const void *const (&ptrs)[N]) {
  for (const void *p : ptrs)
    if (!aligned16(p)) return false;
  return true;
}

bool valid_gate(int kind) { return kind >= HILORE_GATE_NONE && kind <= HILORE_GATE_ELEMENT; }

hilore_status check_shape(int64_t rows, int64_t cols) {
  if (rows < 0 || cols < 0) return HILORE_ERR_INVALID_ARG;
  if (cols % 8 != 0 || cols > hilore::kNormMaxCols || rows >= (int64_t(1) << 31))
    return HILORE_ERR_UNSUPPORTED;
  return HILORE_OK;
}

// ------------------------------------------------------------ block norms --
hilore_status check_block_norm(const hilore_block_norm_desc &d) {
  const hilore_status st = check_shape(d.rows, d.cols);
  if (st != HILORE_OK) return st;
  if (!valid_gate(d.gate_kind)) return HILORE_ERR_INVALID_ARG;
  if (!std::isfinite(d.scale) || !(d.eps >= 0.0f) || !std::isfinite(d.eps))
    return HILORE_ERR_INVALID_ARG;
  if (d.codes && d.cols % 16 != 0) return HILORE_ERR_UNSUPPORTED;
  if (d.rows == 0 || d.cols == 0) return HILORE_OK;  // tensors without elements may be NULL
  if ((d.gate_kind == HILORE_GATE_NONE) != (d.gate == nullptr)) return HILORE_ERR_INVALID_ARG;
  if (!d.y && (d.w_post || d.gate)) return HILORE_ERR_INVALID_ARG;
  if (!d.w_pre && (d.n || d.codes || d.rstd_pre)) return HILORE_ERR_INVALID_ARG;
  if (d.rstd_post && !d.w_post) return HILORE_ERR_INVALID_ARG;
  if ((d.codes == nullptr) != (d.code_scales == nullptr)) return HILORE_ERR_INVALID_ARG;
  if (!d.h && !d.n && !d.codes) return HILORE_ERR_INVALID_ARG;
  if (!d.res || d.ld_res < d.cols || (d.y && d.ld_y < d.cols)) return HILORE_ERR_INVALID_ARG;
  if (d.ld_res % 8 != 0 || (d.y && d.ld_y % 8 != 0)) return HILORE_ERR_ALIGNMENT;
  if (d.h == d.res && d.ld_res != d.cols) return HILORE_ERR_INVALID_ARG;
  const void *ptrs[] = {d.res, d.y, d.w_post, d.gate, d.w_pre, d.h, d.n, d.codes, d.code_scales,
                        d.rstd_post, d.rstd_pre};
  return all_aligned16(ptrs) ? HILORE_OK : HILORE_ERR_ALIGNMENT;
}

bool absent(const hilore_unit_desc &u) { return !u.x && !u.codes; }

// A saved tensor of the backward: rows x cols, bf16 or codes.
hilore_status check_saved(const hilore_unit_desc &u, int64_t rows, int64_t cols, bool scaled) {
  if (absent(u)) return HILORE_OK;
  if (u.rows != rows || u.cols != cols) return HILORE_ERR_INVALID_ARG;
  if (rows == 0 || cols == 0) return HILORE_OK;
  if (u.codes) {
    if (scaled && !u.scales) return HILORE_ERR_INVALID_ARG;
    if (!aligned16(u.codes) || (scaled && !aligned16(u.scales))) return HILORE_ERR_ALIGNMENT;
  } else {
    if (u.ld < cols) return HILORE_ERR_INVALID_ARG;
    if (u.ld % 8 != 0 || !aligned16(u.x)) return HILORE_ERR_ALIGNMENT;
  }
  return HILORE_OK;
}

bool sums_over_rows(const hilore_block_norm_bwd_desc &d) {
  return d.dw_pre || d.dw_post || (d.dgate && d.gate_kind == HILORE_GATE_CHANNEL);
}

hilore_status check_block_norm_bwd(const hilore_block_norm_bwd_desc &d, int code, int block) {
  const hilore_status st = check_shape(d.rows, d.cols);
  if (st != HILORE_OK) return st;
  if (!valid_gate(d.gate_kind) || !std::isfinite(d.scale)) return HILORE_ERR_INVALID_ARG;
  const bool l = d.h.codes || d.y.codes;
  const bool cast = code == HILORE_CODE_FP8_E4M3FN_CAST;
  if (l) {
    const hilore_status cb = check_code_block(code, block);
    if (cb != HILORE_OK) return cb;
    if (!cast && d.cols % block != 0) return HILORE_ERR_UNSUPPORTED;
  }
  if (d.rows == 0 || d.cols == 0) return HILORE_OK;  // tensors without elements may be NULL
  if ((d.gate_kind == HILORE_GATE_NONE) != (d.gate == nullptr)) return HILORE_ERR_INVALID_ARG;
  // what is read follows from what is wanted
  if (!d.dn && (d.w_pre || d.rstd_pre || d.dw_pre)) return HILORE_ERR_INVALID_ARG;
  if (!d.w_post && (d.rstd_post || d.dw_post)) return HILORE_ERR_INVALID_ARG;
  if (d.gate_kind == HILORE_GATE_NONE && d.dgate) return HILORE_ERR_INVALID_ARG;
  if (!d.dn && !d.dh) return HILORE_ERR_INVALID_ARG;
  if (d.dn && (!d.w_pre || !d.rstd_pre || absent(d.h) || d.ld_dn < d.cols))
    return HILORE_ERR_INVALID_ARG;
  if (d.w_post && !d.rstd_post) return HILORE_ERR_INVALID_ARG;
  if ((d.w_post || d.dgate) && absent(d.y)) return HILORE_ERR_INVALID_ARG;
  if (d.dn && d.ld_dn % 8 != 0) return HILORE_ERR_ALIGNMENT;
  const hilore_unit_desc *saved[] = {&d.h, &d.y};
  for (const hilore_unit_desc *u : saved) {
    const hilore_status s = check_saved(*u, d.rows, d.cols, !cast);
    if (s != HILORE_OK) return s;
  }
  const void *ptrs[] = {d.w_post, d.gate, d.w_pre, d.rstd_post, d.rstd_pre, d.dn, d.dh, d.dres,
                        d.dy, d.dw_post, d.dw_pre, d.dgate};
  return all_aligned16(ptrs) ? HILORE_OK : HILORE_ERR_ALIGNMENT;
}

hilore::SavedRows saved_rows(const hilore_unit_desc &u, bool scaled) {
  hilore::SavedRows s{};
  s.codes = static_cast<const uint8_t *>(u.codes);
  s.x = u.codes ? nullptr : u.x;
  s.scales = u.codes && scaled ? u.scales : nullptr;
  s.ld = u.ld;
  return s;
}

// ----------------------------------------------------------- int8 products --
hilore_status check_int8_sizes(const hilore_int8_desc &d) {
  if (d.tokens < 0 || d.k < 0 || d.n < 0) return HILORE_ERR_INVALID_ARG;
  if (d.k % 16 != 0 || d.n % 8 != 0 || d.k > hilore::kInt8MaxK || d.n >= (int64_t(1) << 26) ||
      d.tokens >= (int64_t(1) << 31) || d.tokens * d.n > hilore::kInt8MaxOut)
    return HILORE_ERR_UNSUPPORTED;
  return HILORE_OK;
}

hilore_status check_int8(const hilore_int8_desc &d, bool quantize) {
  const hilore_status sizes = check_int8_sizes(d);
  if (sizes != HILORE_OK) return sizes;
  if (d.tokens == 0 || d.n == 0) return HILORE_OK;
  if (!d.out || d.ldo < d.n) return HILORE_ERR_INVALID_ARG;
  if (d.ldo % 8 != 0) return HILORE_ERR_ALIGNMENT;
  if (!quantize && !d.a_scales) return HILORE_ERR_INVALID_ARG;
  if (d.k > 0) {
    if (!d.w) return HILORE_ERR_INVALID_ARG;
    if (quantize && (!d.x || d.ldx < d.k)) return HILORE_ERR_INVALID_ARG;
    if (!quantize && !d.a) return HILORE_ERR_INVALID_ARG;
    if (quantize && d.ldx % 8 != 0) return HILORE_ERR_ALIGNMENT;
  }
  const void *ptrs[] = {quantize ? d.x : nullptr, quantize ? d.factor : nullptr,
                        quantize ? nullptr : d.a, quantize ? nullptr : d.a_scales,
                        d.w, d.w_scales, d.bias, d.out};
  return all_aligned16(ptrs) ? HILORE_OK : HILORE_ERR_ALIGNMENT;
}

size_t round256(size_t b) { return (b + 255) & ~size_t(255); }

// Workspace of a product: the rounded operand and its scales, then partial sums.
struct Int8Layout {
  size_t off_scales, off_part, bytes;
};

Int8Layout int8_layout(const hilore_int8_desc &d, bool quantize) {
  Int8Layout l{};
  if (quantize) {
    l.off_scales = round256((size_t)d.tokens * (size_t)d.k);
    l.off_part = l.off_scales + round256((size_t)d.tokens * sizeof(float));
  }
  l.bytes = l.off_part + hilore::int8_part_bytes(d.tokens, d.k, d.n);
  return l;
}

hilore_status run_int8(const hilore_int8_desc *d, bool quantize, void *workspace,
                       size_t workspace_bytes, hipStream_t s) {
  if (!d) return HILORE_ERR_INVALID_ARG;
  const hilore_status st = check_int8(*d, quantize);
  if (st != HILORE_OK || d->tokens == 0 || d->n == 0) return st;
  const Int8Layout l = int8_layout(*d, quantize);
  if (l.bytes > 0 && !workspace) return HILORE_ERR_INVALID_ARG;
  if (workspace && !aligned16(workspace)) return HILORE_ERR_ALIGNMENT;
  if (workspace_bytes < l.bytes) return HILORE_ERR_WORKSPACE;
  uint8_t *ws = static_cast<uint8_t *>(workspace);
  hilore::Int8Args a{};
  a.a = d->a;
  a.a_scales = d->a_scales;
  if (quantize) {
    hilore::QuantArgs q{};
    q.x = d->x;
    q.factor = d->factor;
    q.codes = reinterpret_cast<int8_t *>(ws);
    q.scales = reinterpret_cast<float *>(ws + l.off_scales);
    q.tokens = d->tokens;
    q.k = d->k;
    q.ldx = d->ldx;
    const hilore_status qs = hip_status(hilore::launch_quantize_tokens(q, s));
    if (qs != HILORE_OK) return qs;
    a.a = q.codes;
    a.a_scales = q.scales;
  }
  a.w = d->w;
  a.w_scales = d->w_scales;
  a.bias = d->bias;
  a.out = d->out;
  a.tokens = d->tokens;
  a.n = d->n;
  a.ldo = d->ldo;
  a.k = (int)d->k;
  a.out_f32 = d->out_f32 ? 1 : 0;
  a.accumulate = d->accumulate ? 1 : 0;
  a.part = reinterpret_cast<int32_t *>(ws + l.off_part);
  return hip_status(hilore::launch_int8(a, s));
}

// ------------------------------------------------------------------ AdamW --
constexpr int64_t kMaxTensor = int64_t(1) << 32;
constexpr int64_t kMaxElements = int64_t(1) << 40;
// A launch's work-items are counted in 32 bits; 2^23 workgroups of 256 are half of that.
constexpr int64_t kMaxChunks = int64_t(1) << 23;

// Pointers travel to the kernels as 48 bits.
bool fits48(const void *p) { return (reinterpret_cast<uintptr_t>(p) >> 48) == 0; }
uint32_t low32(const void *p) { return (uint32_t)reinterpret_cast<uintptr_t>(p); }
uint32_t upper16(const void *p) { return (uint32_t)((uint64_t)reinterpret_cast<uintptr_t>(p) >> 32); }

hilore_status check_gradients(const hilore_adamw_tensor *t, int n) {
  if (n < 0) return HILORE_ERR_INVALID_ARG;
  if (n == 0) return HILORE_OK;
  if (!t) return HILORE_ERR_INVALID_ARG;
  int64_t total = 0;
  for (int i = 0; i < n; ++i) {
    if (t[i].n < 0) return HILORE_ERR_INVALID_ARG;
    if (t[i].n >= kMaxTensor) return HILORE_ERR_UNSUPPORTED;
    if (t[i].n == 0) continue;
    if (!t[i].grad) return HILORE_ERR_INVALID_ARG;
    if (!aligned16(t[i].grad)) return HILORE_ERR_ALIGNMENT;
    if (!fits48(t[i].grad)) return HILORE_ERR_UNSUPPORTED;
    total += t[i].n;
    if (total > kMaxElements) return HILORE_ERR_UNSUPPORTED;
  }
  return HILORE_OK;
}

hilore_status check_states(const hilore_adamw_tensor *t, int n) {
  for (int i = 0; i < n; ++i) {
    if (!std::isfinite(t[i].lr) || !std::isfinite(t[i].weight_decay)) return HILORE_ERR_INVALID_ARG;
    if (t[i].n == 0) continue;
    if ((!t[i].p && !t[i].p16) || !t[i].m || !t[i].v) return HILORE_ERR_INVALID_ARG;
    if ((t[i].m_scales == nullptr) != (t[i].v_scales == nullptr)) return HILORE_ERR_INVALID_ARG;
    const void *ptrs[] = {t[i].p, t[i].p16, t[i].m, t[i].v};
    if (!all_aligned16(ptrs) || !aligned4(t[i].m_scales) || !aligned4(t[i].v_scales))
      return HILORE_ERR_ALIGNMENT;
    for (const void *p : {(const void *)t[i].p, (const void *)t[i].p16, (const void *)t[i].m, (const void *)t[i].v,
                          (const void *)t[i].m_scales, (const void *)t[i].v_scales})
      if (!fits48(p)) return HILORE_ERR_UNSUPPORTED;
  }
  return HILORE_OK;
}

int64_t norm_chunks(const hilore_adamw_tensor &t) {
  const int64_t elems = hilore::kNormChunkBytes / (t.grad_bf16 ? 2 : 4);
  return (t.n + elems - 1) / elems;
}

void clear(hilore::NormBatch &b, int &count) {
  count = 0;
  b.chunks = 0;
  for (uint32_t &x : b.begin) x = ~0u;
  for (uint32_t &x : b.upper) x = 0;
}

void clear(hilore::AdamwBatch &b, int &count) {
  count = 0;
  b.chunks = 0;
  for (uint32_t &x : b.w) x = 0;
  for (int i = 0; i < b.cap; ++i) b.w[i] = ~0u;
}

}  // namespace

extern "C" {

hilore_status hilore_block_norm(const hilore_block_norm_desc *d, void *stream) {
  if (!d) return HILORE_ERR_INVALID_ARG;
  const hilore_status st = check_block_norm(*d);
  if (st != HILORE_OK || d->rows == 0 || d->cols == 0) return st;
  hilore::BlockNormArgs a{};
  a.res = d->res;
  a.y = d->y;
  a.w_post = d->w_post;
  a.gate = d->gate;
  a.w_pre = d->w_pre;
  a.h = d->h;
  a.n = d->n;
  a.codes = d->codes;
  a.code_scales = d->code_scales;
  a.rstd_post = d->rstd_post;
  a.rstd_pre = d->rstd_pre;
  a.rows = d->rows;
  a.ld_res = d->ld_res;
  a.ld_y = d->ld_y;
  a.cols = (int)d->cols;
  a.scale = d->scale;
  a.eps = d->eps;
  a.inv_cols = (float)(1.0 / (double)d->cols);
  a.gate_kind = d->gate_kind;
  return hip_status(hilore::launch_block_norm(a, static_cast<hipStream_t>(stream)));
}

size_t hilore_block_norm_bwd_workspace_bytes(const hilore_block_norm_bwd_desc *d) {
  if (!d || check_shape(d->rows, d->cols) != HILORE_OK || !sums_over_rows(*d)) return 0;
  return (size_t)3 * (size_t)hilore::block_norm_bwd_groups(d->rows, d->cols, 1) * (size_t)d->cols *
         sizeof(float);
}

hilore_status hilore_block_norm_bwd(const hilore_block_norm_bwd_desc *d, int code, int block,
                                    int accumulate, void *workspace, size_t workspace_bytes,
                                    void *stream) {
  if (!d) return HILORE_ERR_INVALID_ARG;
  const hilore_status st = check_block_norm_bwd(*d, code, block);
  if (st != HILORE_OK || d->cols == 0) return st;
  const size_t need = hilore_block_norm_bwd_workspace_bytes(d);
  if (need > 0 && !workspace) return HILORE_ERR_INVALID_ARG;
  if (workspace && !aligned16(workspace)) return HILORE_ERR_ALIGNMENT;
  if (workspace_bytes < need) return HILORE_ERR_WORKSPACE;
  const bool scaled = code != HILORE_CODE_FP8_E4M3FN_CAST;
  hilore::BlockNormBwdArgs a{};
  // y is read only where its norm or the gate's gradient needs it
  if (d->dn) a.h = saved_rows(d->h, scaled);
  if (d->w_post || d->dgate) a.y = saved_rows(d->y, scaled);
  a.w_post = d->w_post;
  a.gate = d->gate;
  a.w_pre = d->w_pre;
  a.dn = d->dn;
  a.dh = d->dh;
  a.rstd_post = d->rstd_post;
  a.rstd_pre = d->rstd_pre;
  a.dres = d->dres;
  a.dy = d->dy;
  a.dw_post = d->dw_post;
  a.dw_pre = d->dw_pre;
  a.dgate = d->dgate;
  a.rows = d->rows;
  a.ld_dn = d->ld_dn;
  a.cols = (int)d->cols;
  a.scale = d->scale;
  a.inv_cols = (float)(1.0 / (double)d->cols);
  a.gate_kind = d->gate_kind;
  a.accumulate = accumulate ? 1 : 0;
  a.code = code;
  // code and block have been checked only if there is an L unit
  a.block_log2 = (d->h.codes || d->y.codes) && scaled ? __builtin_ctz((unsigned)block) : 0;
  a.sums = sums_over_rows(*d) ? 1 : 0;
  a.groups = hilore::block_norm_bwd_groups(d->rows, d->cols, a.sums);
  a.part = static_cast<float *>(workspace);
  return hip_status(hilore::launch_block_norm_bwd(a, static_cast<hipStream_t>(stream)));
}

size_t hilore_int8_workspace_bytes(const hilore_int8_desc *d, int quantize) {
  if (!d || d->tokens == 0 || d->n == 0 || check_int8_sizes(*d) != HILORE_OK) return 0;
  return int8_layout(*d, quantize != 0).bytes;
}

hilore_status hilore_int8_linear(const hilore_int8_desc *d, void *workspace,
                                 size_t workspace_bytes, void *stream) {
  return run_int8(d, true, workspace, workspace_bytes, static_cast<hipStream_t>(stream));
}

hilore_status hilore_int8_matmul(const hilore_int8_desc *d, void *workspace,
                                 size_t workspace_bytes, void *stream) {
  return run_int8(d, false, workspace, workspace_bytes, static_cast<hipStream_t>(stream));
}

hilore_status hilore_quantize_tokens(const uint16_t *x, const float *factor, int64_t tokens,
                                     int64_t k, int64_t ldx, int8_t *codes, float *scales,
                                     void *stream) {
  if (tokens < 0 || k < 0) return HILORE_ERR_INVALID_ARG;
  if (k % 16 != 0 || k > (int64_t(1) << 30) || tokens >= (int64_t(1) << 31))
    return HILORE_ERR_UNSUPPORTED;
  if (tokens == 0) return HILORE_OK;
  if (!scales || (k > 0 && (!x || !codes || ldx < k))) return HILORE_ERR_INVALID_ARG;
  if (ldx % 8 != 0) return HILORE_ERR_ALIGNMENT;
  const void *ptrs[] = {x, factor, codes, scales};
  if (!all_aligned16(ptrs)) return HILORE_ERR_ALIGNMENT;
  hilore::QuantArgs q{};
  q.x = x;
  q.factor = factor;
  q.codes = codes;
  q.scales = scales;
  q.tokens = tokens;
  q.k = k;
  q.ldx = ldx;
  return hip_status(hilore::launch_quantize_tokens(q, static_cast<hipStream_t>(stream)));
}

size_t hilore_grad_norm_workspace_bytes(const hilore_adamw_tensor *tensors, int n_tensors) {
  if (check_gradients(tensors, n_tensors) != HILORE_OK) return 0;
  int64_t chunks = 0;
  for (int i = 0; i < n_tensors; ++i) chunks += norm_chunks(tensors[i]);
  return (size_t)chunks * sizeof(double);
}

hilore_status hilore_grad_norm(const hilore_adamw_tensor *tensors, int n_tensors, double max_norm,
                               float *norm, void *workspace, size_t workspace_bytes,
                               void *stream) {
  if (!((float)max_norm > 0.0f) || !norm) return HILORE_ERR_INVALID_ARG;
  if (!aligned4(norm)) return HILORE_ERR_ALIGNMENT;
  const hilore_status st = check_gradients(tensors, n_tensors);
  if (st != HILORE_OK) return st;
  const size_t need = hilore_grad_norm_workspace_bytes(tensors, n_tensors);
  if (need > 0 && !workspace) return HILORE_ERR_INVALID_ARG;
  if (workspace && !aligned16(workspace)) return HILORE_ERR_ALIGNMENT;
  if (workspace_bytes < need) return HILORE_ERR_WORKSPACE;
  hipStream_t s = static_cast<hipStream_t>(stream);
  double *part = static_cast<double *>(workspace);
  int64_t done = 0;
  int count = 0;
  hilore::NormBatch b{};
  clear(b, count);
  auto flush = [&]() -> hilore_status {
    if (count == 0) return HILORE_OK;
    b.part = part + done;
    const hilore_status fs = hip_status(hilore::launch_norm_partial(b, s));
    done += b.chunks;
    clear(b, count);
    return fs;
  };
  for (int i = 0; i < n_tensors; ++i) {
    if (tensors[i].n == 0) continue;
    const int64_t chunks = norm_chunks(tensors[i]);
    if (count == hilore::kNormPerLaunch || (count > 0 && b.chunks + chunks > kMaxChunks)) {
      const hilore_status fs = flush();
      if (fs != HILORE_OK) return fs;
    }
    b.grad[count] = low32(tensors[i].grad) | (tensors[i].grad_bf16 ? 1u : 0u);
    b.n[count] = (uint32_t)tensors[i].n;
    b.upper[count / 2] |= upper16(tensors[i].grad) << (16 * (count & 1));
    b.begin[count++] = b.chunks;
    b.chunks += (uint32_t)chunks;
  }
  const hilore_status fs = flush();
  if (fs != HILORE_OK) return fs;
  return hip_status(hilore::launch_norm_fold(part, done, (float)max_norm, norm, s));
}

hilore_status hilore_adamw(const hilore_adamw_tensor *tensors, int n_tensors, double beta1,
                           double beta2, double eps, int64_t step, const float *norm,
                           uint32_t seed, void *stream) {
  if (!(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) || step < 1)
    return HILORE_ERR_INVALID_ARG;
  if (!((float)eps >= FLT_MIN) || !std::isfinite((float)eps)) return HILORE_ERR_INVALID_ARG;
  hilore_status st = check_gradients(tensors, n_tensors);
  if (st != HILORE_OK) return st;
  st = check_states(tensors, n_tensors);
  if (st != HILORE_OK) return st;
  if (!aligned4(norm)) return HILORE_ERR_ALIGNMENT;
  const double c1 = 1.0 - std::pow(beta1, (double)step);
  const double c2 = 1.0 - std::pow(beta2, (double)step);
  hipStream_t s = static_cast<hipStream_t>(stream);
  hilore::AdamwBatch b;
  b.norm = norm;
  b.beta1 = (float)beta1;
  b.one_beta1 = (float)(1.0 - beta1);
  b.beta2 = (float)beta2;
  b.one_beta2 = (float)(1.0 - beta2);
  b.eps = (float)eps;
  b.inv_sqrt_c2 = (float)(1.0 / std::sqrt(c2));
  b.seed = seed;
  bool has_p = false, has_p16 = false, has_scales = false;
  for (int i = 0; i < n_tensors; ++i) {
    if (tensors[i].n == 0) continue;
    has_p |= tensors[i].p != nullptr;
    has_p16 |= tensors[i].p16 != nullptr;
    has_scales |= tensors[i].m_scales != nullptr;
  }
  b.has_p = has_p;
  b.has_p16 = has_p16;
  b.stride = 9 + (has_p && has_p16 ? 2 : 0) + (has_scales ? 3 : 0);
  b.cap = hilore::adamw_capacity(b.stride);
  int count;
  clear(b, count);
  // one without elements keeps its number and gets no workgroup
  for (int i = 0; i < n_tensors; ++i) {
    const hilore_adamw_tensor &t = tensors[i];
    const int64_t chunks = (t.n + hilore::kAdamwChunk - 1) / hilore::kAdamwChunk;
    if (count == b.cap || (b.chunks > 0 && b.chunks + chunks > kMaxChunks)) {
      if (b.chunks > 0) {
        st = hip_status(hilore::launch_adamw(b, s));
        if (st != HILORE_OK) return st;
      }
      clear(b, count);
    }
    if (count == 0) b.first = i;
    uint32_t *rec = b.w + b.cap + count * b.stride;
    if (t.n > 0) {
      rec[0] = low32(t.grad) | (t.grad_bf16 ? 1u : 0u);
      rec[1] = low32(t.m);
      rec[2] = low32(t.v);
      rec[3] = upper16(t.grad) | upper16(t.m) << 16;
      rec[4] = (uint32_t)t.n;
      const void *param = has_p ? (const void *)t.p : t.p16;
      rec[5] = upper16(t.v) | upper16(param) << 16;
      rec[6] = low32(param);
      rec[7] = __builtin_bit_cast(uint32_t, (float)((double)t.lr / c1));
      rec[8] = __builtin_bit_cast(uint32_t, (float)(1.0 - (double)t.lr * (double)t.weight_decay));
      uint32_t *next = rec + 9;
      if (has_p && has_p16) {
        *next++ = low32(t.p16);
        *next++ = upper16(t.p16);
      }
      if (has_scales) {
        *next++ = low32(t.m_scales);
        *next++ = low32(t.v_scales);
        *next = upper16(t.m_scales) | upper16(t.v_scales) << 16;
      }
    }
    b.w[count++] = b.chunks;
    b.chunks += (uint32_t)chunks;
  }
  return b.chunks > 0 ? hip_status(hilore::launch_adamw(b, s)) : HILORE_OK;
}

}  // extern "C"
