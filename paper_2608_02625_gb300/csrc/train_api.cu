// libdlmrefine C ABI: the entry points of training the refiner's last layer
// (argument validation, dispatch). The rules of the other entry points hold: a
// nonzero status means that nothing was launched, unless a launch itself failed.
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <new>
#include <vector>

#include "dlm_checks.h"
#include "dlm_internal.h"
#include "dlmrefine.h"

namespace {

using namespace dlm;

// Rows of a [N, d] or [B, L, d] tensor: their number, width and (even) stride.
int rows_of(const dlm_tensor* t, const char* name, int dtype_mask, int64_t* N, int64_t* d, int64_t* stride) {
  int st;
  if ((st = check_tensor(t, name, dtype_mask, 2, 3))) return st;
  const int nd = t->ndim;
  *d = t->shape[nd - 1];
  *N = 1;
  for (int i = 0; i < nd - 1; ++i) *N *= t->shape[i];
  *stride = t->stride[nd - 2];
  if (nd == 3 && t->shape[1] == 1) *stride = t->stride[0];
  if (*N > 0x7FFFFFFFLL) return fail(DLM_ERR_SHAPE, "%s: more than 2^31 - 1 rows", name);
  if (nd == 3 && t->shape[0] > 1 && t->shape[1] > 1 && t->stride[0] != t->shape[1] * t->stride[1])
    return fail(DLM_ERR_STRIDE, "%s: rows must be evenly strided ([B, L, d] with stride[0] = L * stride[1])", name);
  if (*N > 1 && *d > 0 && *stride < *d) return fail(DLM_ERR_STRIDE, "%s: rows overlap", name);
  if (*N <= 1) *stride = *d;
  return DLM_OK;
}

bool same_shape(const dlm_tensor* a, const dlm_tensor* b) {
  if (a->ndim != b->ndim) return false;
  for (int i = 0; i < a->ndim; ++i)
    if (a->shape[i] != b->shape[i]) return false;
  return true;
}

// A vector of n contiguous entries, any rank; null allowed where `optional`.
int check_vector(const dlm_tensor* t, const char* name, int dtype_mask, int64_t n, bool optional) {
  if (!t && optional) return DLM_OK;
  int st;
  if ((st = check_tensor(t, name, dtype_mask, 1, 3))) return st;
  if (numel(t) != n) return fail(DLM_ERR_SHAPE, "%s: %lld entries expected", name, (long long)n);
  if (!is_dense(t)) return fail(DLM_ERR_STRIDE, "%s must be contiguous", name);
  return DLM_OK;
}

// Bytes between the rows of a tensor whose rows are evenly strided; 0 for a vector or a single row.
int64_t row_pitch(const dlm_tensor* t) {
  if (t->ndim < 2 || numel(t) <= t->shape[t->ndim - 1]) return 0;
  return (t->ndim == 3 && t->shape[1] == 1 ? t->stride[0] : t->stride[t->ndim - 2]) * elem_size(t->dtype);
}

// As overlaps(), of tensors with evenly strided rows, but the rows of one may lie between those of
// the other (column ranges of one buffer).
bool rows_overlap(const dlm_tensor* a, const dlm_tensor* b) {
  if (!overlaps(a, b)) return false;
  const int64_t pitch = row_pitch(a);
  if (pitch == 0 || pitch != row_pitch(b)) return true;
  const auto width = [](const dlm_tensor* t) { return t->shape[t->ndim - 1] * elem_size(t->dtype); };
  const intptr_t apart = static_cast<intptr_t>(reinterpret_cast<uintptr_t>(b->data) - reinterpret_cast<uintptr_t>(a->data));
  const int64_t at = (apart % pitch + pitch) % pitch;  // where b's rows start in a's pitch
  return at < width(a) || at + width(b) > pitch;
}

// No output may overlap an input or another output. Null descriptors are skipped.
int check_disjoint(const dlm_tensor* const* outs, int n_outs, const dlm_tensor* const* ins, int n_ins,
                   bool (*overlap)(const dlm_tensor*, const dlm_tensor*) = overlaps) {
  for (int i = 0; i < n_outs; ++i) {
    if (!outs[i]) continue;
    for (int j = 0; j < n_ins; ++j)
      if (ins[j] && overlap(outs[i], ins[j])) return fail(DLM_ERR_ARG, "an output overlaps an input");
    for (int j = 0; j < i; ++j)
      if (outs[j] && overlap(outs[i], outs[j])) return fail(DLM_ERR_ARG, "outputs overlap each other");
  }
  return DLM_OK;
}

// The caller's workspace: present, aligned, large enough and apart from every tensor.
int check_workspace(const void* workspace, size_t bytes, size_t need, uintptr_t align, const dlm_tensor* const* all, int n) {
  if (need == 0) return DLM_OK;
  if (!workspace) return fail(DLM_ERR_NULL, "workspace is NULL");
  if (reinterpret_cast<uintptr_t>(workspace) % align != 0)
    return fail(DLM_ERR_ALIGN, "workspace not %d-byte aligned", static_cast<int>(align));
  if (bytes < need) return fail(DLM_ERR_ARG, "workspace too small: %zu bytes, %zu needed", bytes, need);
  const uintptr_t wlo = reinterpret_cast<uintptr_t>(workspace), whi = wlo + need;
  for (int i = 0; i < n; ++i) {
    if (!all[i] || numel(all[i]) == 0) continue;
    uintptr_t lo, hi;
    byte_span(all[i], &lo, &hi);
    if (lo < whi && wlo < hi) return fail(DLM_ERR_ARG, "workspace overlaps a tensor");
  }
  return DLM_OK;
}

struct Span {
  uintptr_t lo, hi;
};

// Whether no written range overlaps another range: both lists walked together in the order of
// their addresses (which tensors allocated one after another often have already).
bool written_apart(std::vector<Span>* read, std::vector<Span>* written) {
  const auto before = [](const Span& p, const Span& q) { return p.lo < q.lo; };
  for (std::vector<Span>* v : {read, written})
    if (!std::is_sorted(v->begin(), v->end(), before)) std::sort(v->begin(), v->end(), before);
  uintptr_t end = 0, written_end = 0;  // the furthest end so far, of any and of a written range
  for (size_t i = 0, j = 0; i < read->size() || j < written->size();) {
    const bool write = i == read->size() || (j < written->size() && (*written)[j].lo < (*read)[i].lo);
    const Span& p = write ? (*written)[j++] : (*read)[i++];
    if (p.lo < (write ? end : written_end)) return false;
    end = std::max(end, p.hi);
    if (write) written_end = std::max(written_end, p.hi);
  }
  return true;
}

constexpr int64_t kMostElements = int64_t{1} << 40;  // of a tensor in a list (a flat buffer is one extent)

// A contiguous tensor of a list, and the bytes that it takes (none where it is empty).
int list_tensor(const dlm_tensor* t, const char* name, int dtype_mask, int i, Span* span) {
  int st;
  if ((st = check_tensor(t, name, dtype_mask, 1, 4, kMostElements))) return st;
  if (numel(t) > kMostElements) return fail(DLM_ERR_SHAPE, "%s %d: more than 2^40 elements", name, i);
  if (!is_dense(t)) return fail(DLM_ERR_STRIDE, "%s %d must be contiguous", name, i);
  span->lo = reinterpret_cast<uintptr_t>(t->data);
  span->hi = span->lo + static_cast<uintptr_t>(numel(t)) * elem_size(t->dtype);
  return DLM_OK;
}

// Every kernel records device-side failures in the error word; refuse to launch without it.
int require_error_word() {
  if (!device_error_word()) return fail(DLM_ERR_CUDA, "device error word unavailable on this device");
  return DLM_OK;
}

constexpr int64_t kMostNormWidth = int64_t{1} << 24;

bool aligned_rows(const dlm_tensor* t) {
  if (reinterpret_cast<uintptr_t>(t->data) % 16 != 0) return false;
  return t->shape[0] <= 1 || (t->stride[0] * elem_size(t->dtype)) % 16 == 0;
}

// A matrix that TMA moves: even rows at multiples of 16 bytes, less than 2^40 bytes apart.
int check_matrix(const dlm_tensor* t, const char* name, int64_t rows, int64_t width) {
  if (rows > 1 && t->stride[0] < width) return fail(DLM_ERR_STRIDE, "%s rows overlap", name);
  if (rows > 1 && t->stride[0] >= (int64_t{1} << 40) / elem_size(t->dtype))
    return fail(DLM_ERR_STRIDE, "%s rows must lie less than 2^40 bytes apart", name);
  if (!aligned_rows(t)) return fail(DLM_ERR_ALIGN, "%s rows must start at multiples of 16 bytes", name);
  return DLM_OK;
}

constexpr int64_t kMostRows = int64_t{1} << 28, kMostVocab = int64_t{1} << 30, kMostWidth = int64_t{1} << 20;

// The arguments that the loss and its gradients share.
int prepare_loss(const dlm_tensor* hidden, const dlm_tensor* weight, const dlm_tensor* targets, LossArgs* a) {
  int st;
  if ((st = rows_of(hidden, "hidden", 1 << DLM_BF16, &a->N, &a->d, &a->s_hidden))) return st;
  if ((st = check_tensor(weight, "weight", 1 << DLM_BF16, 2, 2))) return st;
  if ((st = check_vector(targets, "targets", 1 << DLM_I32, a->N, false))) return st;
  a->V = weight->shape[0];
  if (weight->shape[1] != a->d) return fail(DLM_ERR_SHAPE, "weight must be [V, d] with the d of hidden");
  if (a->d < 8 || a->d % 8 != 0) return fail(DLM_ERR_SHAPE, "d must be a positive multiple of 8 (got %lld)", (long long)a->d);
  if (a->V < 1) return fail(DLM_ERR_SHAPE, "V must be >= 1");
  if (a->N > kMostRows || a->V > kMostVocab || a->d > kMostWidth)
    return fail(DLM_ERR_SHAPE, "at most 2^28 rows, 2^30 tokens and a width of 2^20");
  if ((st = check_matrix(weight, "weight", a->V, a->d))) return st;
  a->hidden = hidden->data;
  a->weight = weight->data;
  a->targets = static_cast<const int32_t*>(targets->data);
  a->s_weight = a->V > 1 ? weight->stride[0] : a->d;
  return DLM_OK;
}

// A [N, width] or [B, L, width] tensor of bf16 rows (null allowed where `optional`: `to` is
// left empty). aligned: as TMA and 16-byte loads take it.
int block_rows(const dlm_tensor* t, const char* name, bool optional, bool aligned, Matrix* to) {
  if (!t && optional) return DLM_OK;
  int st;
  int64_t N, width, stride;
  if ((st = rows_of(t, name, 1 << DLM_BF16, &N, &width, &stride))) return st;
  if (N > kMostRows || width > kMostWidth) return fail(DLM_ERR_SHAPE, "%s: at most 2^28 rows and a width of 2^20", name);
  if (N * width > kMostElements) return fail(DLM_ERR_SHAPE, "%s: more than 2^40 elements", name);
  if (width < 8 || width % 8 != 0) return fail(DLM_ERR_SHAPE, "%s: the width must be a positive multiple of 8 (got %lld)", name, (long long)width);
  if (stride >= (int64_t{1} << 39)) return fail(DLM_ERR_STRIDE, "%s rows must lie less than 2^40 bytes apart", name);
  if (aligned && N > 0 && (reinterpret_cast<uintptr_t>(t->data) % 16 != 0 || stride % 8 != 0))
    return fail(DLM_ERR_ALIGN, "%s rows must start at multiples of 16 bytes", name);
  *to = {t->data, N, width, stride};
  return DLM_OK;
}

// A [rows, width] weight, or its gradient.
int block_weight(const dlm_tensor* t, const char* name, int64_t width, bool optional, Matrix* to) {
  if (!t && optional) return DLM_OK;
  int st;
  if ((st = check_tensor(t, name, 1 << DLM_BF16, 2, 2))) return st;
  const int64_t rows = t->shape[0];
  if (t->shape[1] != width) return fail(DLM_ERR_SHAPE, "%s must have the width of x", name);
  if (rows < 8 || rows % 8 != 0 || rows > kMostWidth)
    return fail(DLM_ERR_SHAPE, "%s: a multiple of 8 rows up to 2^20 expected (got %lld)", name, (long long)rows);
  if ((st = check_matrix(t, name, rows, width))) return st;
  *to = {t->data, rows, width, t->stride[0]};
  return DLM_OK;
}

int check_act(int32_t act) {
  if (act < DLM_ACT_NONE || act > DLM_ACT_GELU) return fail(DLM_ERR_ARG, "unknown activation %d", act);
  return DLM_OK;
}

// Rows of the leading shape of x and a width of their own.
int check_like(const Matrix& t, const dlm_tensor* desc, const char* name, const dlm_tensor* x, int64_t width) {
  if (!desc) return DLM_OK;
  bool same = desc->ndim == x->ndim && t.cols == width;
  for (int i = 0; same && i < x->ndim - 1; ++i) same = desc->shape[i] == x->shape[i];
  if (!same) return fail(DLM_ERR_SHAPE, "%s must have the rows of x and a width of %lld", name, (long long)width);
  return DLM_OK;
}

// The gradient of no rows.
int zero_matrix(const Matrix& t) {
  if (!t.data) return DLM_OK;
  const cudaError_t e = cudaMemset2DAsync(t.data, static_cast<size_t>(t.stride) * 2, 0, static_cast<size_t>(t.cols) * 2,
                                          static_cast<size_t>(t.rows), current_stream());
  return e == cudaSuccess ? DLM_OK : fail(DLM_ERR_CUDA, "gradient of no rows: %s", cudaGetErrorString(e));
}

bool block_sizes(int64_t rows, int64_t a, int64_t b) {
  const auto width = [](int64_t w) { return w >= 8 && w % 8 == 0 && w <= kMostWidth; };
  return rows > 0 && rows <= kMostRows && width(a) && width(b) && rows * a <= kMostElements && rows * b <= kMostElements;
}

}  // namespace

extern "C" {

int dlm_gated_linear(const dlm_tensor* x, const dlm_tensor* w_gate, const dlm_tensor* w_up, int32_t act, dlm_tensor* out,
                     dlm_tensor* gate, dlm_tensor* up) {
  clear_error();
  GatedArgs a = {};
  int st;
  if ((st = block_rows(x, "x", false, true, &a.x))) return st;
  if ((st = block_weight(w_gate, "w_gate", a.x.cols, false, &a.w_gate))) return st;
  if ((st = block_weight(w_up, "w_up", a.x.cols, false, &a.w_up))) return st;
  if (!same_shape(w_gate, w_up)) return fail(DLM_ERR_SHAPE, "w_up must have the shape of w_gate");
  if ((st = check_act(act))) return st;
  if ((st = block_rows(out, "out", false, true, &a.out))) return st;
  if ((gate == nullptr) != (up == nullptr)) return fail(DLM_ERR_NULL, "gate and up must both be given or both be NULL");
  if ((st = block_rows(gate, "gate", true, true, &a.gate))) return st;
  if ((st = block_rows(up, "up", true, true, &a.up))) return st;
  if ((st = check_like(a.out, out, "out", x, a.w_gate.rows))) return st;
  if ((st = check_like(a.gate, gate, "gate", x, a.w_gate.rows))) return st;
  if ((st = check_like(a.up, up, "up", x, a.w_gate.rows))) return st;
  const dlm_tensor* outs[3] = {out, gate, up};
  const dlm_tensor* ins[3] = {x, w_gate, w_up};
  if ((st = check_disjoint(outs, 3, ins, 3, rows_overlap))) return st;
  if (a.x.rows == 0) return DLM_OK;
  if ((st = require_error_word())) return st;
  a.act = act;
  return launch_gated(a, current_stream());
}

size_t dlm_gated_linear_grad_workspace_bytes(int64_t rows, int64_t f, int64_t d) {
  return block_sizes(rows, f, d) ? gated_grad_workspace_bytes(rows, f, d) : 0;
}

int dlm_gated_linear_grad(const dlm_tensor* dout, const dlm_tensor* x, const dlm_tensor* w_gate, const dlm_tensor* w_up,
                          const dlm_tensor* gate, const dlm_tensor* up, int32_t act, const dlm_tensor* add, dlm_tensor* dx,
                          dlm_tensor* dw_gate, dlm_tensor* dw_up, void* workspace, size_t workspace_bytes) {
  clear_error();
  GatedArgs a = {};
  Matrix m_add = {}, m_dx = {};
  int st;
  if ((st = block_rows(x, "x", false, true, &a.x))) return st;
  if ((st = block_weight(w_gate, "w_gate", a.x.cols, false, &a.w_gate))) return st;
  if ((st = block_weight(w_up, "w_up", a.x.cols, false, &a.w_up))) return st;
  if (!same_shape(w_gate, w_up)) return fail(DLM_ERR_SHAPE, "w_up must have the shape of w_gate");
  if ((st = check_act(act))) return st;
  if ((st = block_rows(dout, "dout", false, true, &a.dout))) return st;
  if ((st = block_rows(gate, "gate", false, true, &a.gate))) return st;
  if ((st = block_rows(up, "up", false, true, &a.up))) return st;
  if ((st = check_like(a.dout, dout, "dout", x, a.w_gate.rows))) return st;
  if ((st = check_like(a.gate, gate, "gate", x, a.w_gate.rows))) return st;
  if ((st = check_like(a.up, up, "up", x, a.w_gate.rows))) return st;
  if (add && !dx) return fail(DLM_ERR_NULL, "add is given, dx is NULL");
  if ((st = block_rows(add, "add", true, false, &m_add))) return st;
  if ((st = block_rows(dx, "dx", true, false, &m_dx))) return st;
  if ((st = check_like(m_add, add, "add", x, a.x.cols))) return st;
  if ((st = check_like(m_dx, dx, "dx", x, a.x.cols))) return st;
  if ((dw_gate == nullptr) != (dw_up == nullptr)) return fail(DLM_ERR_NULL, "dw_gate and dw_up must both be given or both be NULL");
  if (!dx && !dw_gate) return fail(DLM_ERR_NULL, "dx, dw_gate and dw_up are all NULL");
  if ((st = block_weight(dw_gate, "dw_gate", a.x.cols, true, &a.dw_gate))) return st;
  if ((st = block_weight(dw_up, "dw_up", a.x.cols, true, &a.dw_up))) return st;
  if (dw_gate && (!same_shape(w_gate, dw_gate) || !same_shape(w_gate, dw_up)))
    return fail(DLM_ERR_SHAPE, "dw_gate and dw_up must have the shape of w_gate");
  const dlm_tensor* outs[3] = {dx, dw_gate, dw_up};
  const dlm_tensor* ins[7] = {dout, x, w_gate, w_up, gate, up, add && dx && same_view(add, dx) ? nullptr : add};
  if ((st = check_disjoint(outs, 3, ins, 7, rows_overlap))) return st;
  if (a.x.rows == 0) return (st = zero_matrix(a.dw_gate)) ? st : zero_matrix(a.dw_up);
  const dlm_tensor* all[10] = {dout, x, w_gate, w_up, gate, up, add, dx, dw_gate, dw_up};
  const size_t need = gated_grad_workspace_bytes(a.x.rows, a.w_gate.rows, a.x.cols);
  if ((st = check_workspace(workspace, workspace_bytes, need, 16, all, 10))) return st;
  if ((st = require_error_word())) return st;
  a.act = act;
  a.add = m_add.data;
  a.s_add = m_add.stride;
  a.dx = m_dx.data;
  a.s_dx = m_dx.stride;
  a.workspace = workspace;
  return launch_gated_grad(a, current_stream());
}

size_t dlm_linear_workspace_bytes(int64_t rows, int64_t m, int64_t k) {
  return block_sizes(rows, m, k) ? linear_workspace_bytes(rows, m, k) : 0;
}

int dlm_linear(const dlm_tensor* x, const dlm_tensor* weight, const dlm_tensor* bias, int32_t act, const dlm_tensor* residual,
               dlm_tensor* out, dlm_tensor* pre, void* workspace, size_t workspace_bytes) {
  clear_error();
  LinearArgs a = {};
  Matrix m_out = {}, m_residual = {}, m_pre = {};
  int st;
  if ((st = block_rows(x, "x", false, true, &a.x))) return st;
  if ((st = block_weight(weight, "weight", a.x.cols, false, &a.w))) return st;
  if ((st = check_vector(bias, "bias", kMaskBF16F32, a.w.rows, true))) return st;
  if ((st = check_act(act))) return st;
  if ((st = block_rows(residual, "residual", true, false, &m_residual))) return st;
  if ((st = block_rows(out, "out", false, false, &m_out))) return st;
  if ((st = block_rows(pre, "pre", true, false, &m_pre))) return st;
  if ((st = check_like(m_residual, residual, "residual", x, a.w.rows))) return st;
  if ((st = check_like(m_out, out, "out", x, a.w.rows))) return st;
  if ((st = check_like(m_pre, pre, "pre", x, a.w.rows))) return st;
  const dlm_tensor* outs[2] = {out, pre};
  const dlm_tensor* ins[4] = {x, weight, bias, nullptr};
  if ((st = check_disjoint(outs, 2, ins, 4, rows_overlap))) return st;
  if (residual && ((!same_view(residual, out) && rows_overlap(residual, out)) || (pre && rows_overlap(residual, pre))))
    return fail(DLM_ERR_ARG, "an output overlaps an input");
  if (a.x.rows == 0) return DLM_OK;
  const dlm_tensor* all[6] = {x, weight, bias, residual, out, pre};
  if ((st = check_workspace(workspace, workspace_bytes, linear_workspace_bytes(a.x.rows, a.w.rows, a.x.cols), 16, all, 6))) return st;
  if ((st = require_error_word())) return st;
  a.ep = {act, bias ? bias->data : nullptr, bias && bias->dtype == DLM_BF16, m_residual.data, m_out.data, m_pre.data,
          m_residual.stride, m_out.stride, m_pre.stride};
  a.workspace = workspace;
  return launch_linear(a, current_stream());
}

size_t dlm_linear_grad_workspace_bytes(int64_t rows, int64_t m, int64_t k) {
  return block_sizes(rows, m, k) ? linear_grad_workspace_bytes(rows, m, k) : 0;
}

int dlm_linear_grad(const dlm_tensor* dout, const dlm_tensor* x, const dlm_tensor* weight, const dlm_tensor* pre, int32_t act,
                    const dlm_tensor* add, dlm_tensor* dx, dlm_tensor* dweight, dlm_tensor* dbias, void* workspace,
                    size_t workspace_bytes) {
  clear_error();
  LinearArgs a = {};
  Matrix m_add = {}, m_dx = {};
  int st;
  if ((st = block_rows(x, "x", false, true, &a.x))) return st;
  if ((st = block_weight(weight, "weight", a.x.cols, false, &a.w))) return st;
  if ((st = check_act(act))) return st;
  if ((st = block_rows(dout, "dout", false, true, &a.dout))) return st;
  if ((act == DLM_ACT_NONE) != (pre == nullptr))
    return fail(pre ? DLM_ERR_ARG : DLM_ERR_NULL, "pre belongs to an activation, and is needed with one");
  if ((st = block_rows(pre, "pre", true, true, &a.pre))) return st;
  if ((st = check_like(a.dout, dout, "dout", x, a.w.rows))) return st;
  if ((st = check_like(a.pre, pre, "pre", x, a.w.rows))) return st;
  if (add && !dx) return fail(DLM_ERR_NULL, "add is given, dx is NULL");
  if ((st = block_rows(add, "add", true, false, &m_add))) return st;
  if ((st = block_rows(dx, "dx", true, false, &m_dx))) return st;
  if ((st = check_like(m_add, add, "add", x, a.x.cols))) return st;
  if ((st = check_like(m_dx, dx, "dx", x, a.x.cols))) return st;
  if (!dx && !dweight && !dbias) return fail(DLM_ERR_NULL, "dx, dweight and dbias are all NULL");
  if ((st = block_weight(dweight, "dweight", a.x.cols, true, &a.dw))) return st;
  if (dweight && !same_shape(weight, dweight)) return fail(DLM_ERR_SHAPE, "dweight must have the shape of weight");
  if ((st = check_vector(dbias, "dbias", kMaskBF16F32, a.w.rows, true))) return st;
  const dlm_tensor* outs[3] = {dx, dweight, dbias};
  const dlm_tensor* ins[5] = {dout, x, weight, pre, add && dx && same_view(add, dx) ? nullptr : add};
  if ((st = check_disjoint(outs, 3, ins, 5, rows_overlap))) return st;
  if (a.x.rows == 0) {
    if ((st = zero_matrix(a.dw)) || !dbias) return st;
    const cudaError_t e = cudaMemsetAsync(dbias->data, 0, static_cast<size_t>(a.w.rows * elem_size(dbias->dtype)), current_stream());
    return e == cudaSuccess ? DLM_OK : fail(DLM_ERR_CUDA, "gradient of no rows: %s", cudaGetErrorString(e));
  }
  const dlm_tensor* all[8] = {dout, x, weight, pre, add, dx, dweight, dbias};
  const size_t need = linear_grad_workspace_bytes(a.x.rows, a.w.rows, a.x.cols);
  if ((st = check_workspace(workspace, workspace_bytes, need, 16, all, 8))) return st;
  if ((st = require_error_word())) return st;
  a.ep.act = act;
  a.ep.bias_bf16 = dbias && dbias->dtype == DLM_BF16;
  a.ep.residual = m_add.data;
  a.ep.s_residual = m_add.stride;
  a.ep.out = m_dx.data;
  a.ep.s_out = m_dx.stride;
  a.dbias = dbias ? dbias->data : nullptr;
  a.workspace = workspace;
  return launch_linear_grad(a, current_stream());
}

size_t dlm_lmhead_loss_workspace_bytes(int64_t rows, int64_t d) {
  return rows > 0 && rows <= kMostRows && d > 0 && d <= kMostWidth ? loss_workspace_bytes(rows, d) : 0;
}

int dlm_lmhead_loss(const dlm_tensor* hidden, const dlm_tensor* weight, const dlm_tensor* targets, dlm_tensor* loss,
                    dlm_tensor* lse, void* workspace, size_t workspace_bytes) {
  clear_error();
  LossArgs a = {};
  int st;
  if ((st = prepare_loss(hidden, weight, targets, &a))) return st;
  if ((st = check_vector(loss, "loss", 1 << DLM_F32, a.N, false))) return st;
  if ((st = check_vector(lse, "lse", 1 << DLM_F32, a.N, false))) return st;
  const dlm_tensor* outs[2] = {loss, lse};
  const dlm_tensor* ins[3] = {hidden, weight, targets};
  if ((st = check_disjoint(outs, 2, ins, 3))) return st;
  if (a.N == 0) return DLM_OK;
  const dlm_tensor* all[5] = {hidden, weight, targets, loss, lse};
  if ((st = check_workspace(workspace, workspace_bytes, loss_workspace_bytes(a.N, a.d), 16, all, 5))) return st;
  if ((st = require_error_word())) return st;
  a.loss = static_cast<float*>(loss->data);
  a.lse_out = static_cast<float*>(lse->data);
  a.workspace = workspace;
  return launch_loss(a, current_stream());
}

size_t dlm_lmhead_loss_grad_workspace_bytes(int64_t rows, int64_t vocab, int64_t d, int64_t piece) {
  const bool fine = rows > 0 && rows <= kMostRows && vocab > 0 && vocab <= kMostVocab && d > 0 && d <= kMostWidth && piece >= 0;
  return fine ? loss_grad_workspace_bytes(rows, vocab, d, piece) : 0;
}

int dlm_lmhead_loss_grad(const dlm_tensor* hidden, const dlm_tensor* weight, const dlm_tensor* targets, const dlm_tensor* lse,
                         const dlm_tensor* dloss, dlm_tensor* d_hidden, dlm_tensor* d_weight, void* workspace,
                         size_t workspace_bytes) {
  clear_error();
  LossArgs a = {};
  int64_t N2, d2;
  int st;
  if ((st = prepare_loss(hidden, weight, targets, &a))) return st;
  if ((st = check_vector(lse, "lse", 1 << DLM_F32, a.N, false))) return st;
  if ((st = check_vector(dloss, "dloss", 1 << DLM_F32, a.N, false))) return st;
  if (!d_hidden && !d_weight) return fail(DLM_ERR_NULL, "d_hidden and d_weight are both NULL");
  if (d_hidden) {
    if ((st = rows_of(d_hidden, "d_hidden", 1 << DLM_BF16, &N2, &d2, &a.s_dhidden))) return st;
    if (!same_shape(hidden, d_hidden)) return fail(DLM_ERR_SHAPE, "d_hidden must have the shape of hidden");
    a.d_hidden = d_hidden->data;
  }
  if (d_weight) {
    if ((st = check_tensor(d_weight, "d_weight", 1 << DLM_BF16, 2, 2))) return st;
    if (!same_shape(weight, d_weight)) return fail(DLM_ERR_SHAPE, "d_weight must have the shape of weight");
    if ((st = check_matrix(d_weight, "d_weight", a.V, a.d))) return st;
    a.d_weight = d_weight->data;
    a.s_dweight = a.V > 1 ? d_weight->stride[0] : a.d;
  }
  const dlm_tensor* outs[2] = {d_hidden, d_weight};
  const dlm_tensor* ins[5] = {hidden, weight, targets, lse, dloss};
  if ((st = check_disjoint(outs, 2, ins, 5))) return st;
  if (a.N == 0) {  // the gradient of no rows
    if (!d_weight) return DLM_OK;
    const cudaError_t e = cudaMemset2DAsync(a.d_weight, static_cast<size_t>(a.s_dweight) * 2, 0, static_cast<size_t>(a.d) * 2,
                                            static_cast<size_t>(a.V), current_stream());
    return e == cudaSuccess ? DLM_OK : fail(DLM_ERR_CUDA, "d_weight: %s", cudaGetErrorString(e));
  }
  const dlm_tensor* all[7] = {hidden, weight, targets, lse, dloss, d_hidden, d_weight};
  // At least pieces of 256 columns; all that is given is used, up to the whole vocabulary.
  const size_t most = loss_grad_workspace_bytes(a.N, a.V, a.d, a.V), least = loss_grad_workspace_bytes(a.N, a.V, a.d, 256);
  if ((st = check_workspace(workspace, workspace_bytes, least, 16, nullptr, 0))) return st;
  a.workspace_bytes = workspace_bytes < most ? workspace_bytes : most;
  if ((st = check_workspace(workspace, workspace_bytes, a.workspace_bytes, 16, all, 7))) return st;
  if ((st = require_error_word())) return st;
  a.lse = static_cast<const float*>(lse->data);
  a.dloss = static_cast<const float*>(dloss->data);
  a.workspace = workspace;
  return launch_loss_grad(a, current_stream());
}

int dlm_layer_norm(const dlm_tensor* x, const dlm_tensor* weight, const dlm_tensor* bias, float eps, dlm_tensor* out,
                   dlm_tensor* mean, dlm_tensor* rstd) {
  clear_error();
  NormArgs a = {};
  int64_t N2, d2;
  int st;
  if ((st = rows_of(x, "x", kMaskBF16F32, &a.N, &a.d, &a.s_x))) return st;
  if ((st = rows_of(out, "out", 1 << x->dtype, &N2, &d2, &a.s_out))) return st;
  if (!same_shape(x, out)) return fail(DLM_ERR_SHAPE, "out must have the shape of x");
  if (a.d < 1 || a.d > kMostNormWidth) return fail(DLM_ERR_SHAPE, "rows must have between 1 and 2^24 elements");
  if ((st = check_vector(weight, "weight", kMaskBF16F32, a.d, false))) return st;
  if ((st = check_vector(bias, "bias", 1 << weight->dtype, a.d, true))) return st;
  if ((st = check_vector(mean, "mean", 1 << DLM_F32, a.N, true))) return st;
  if ((st = check_vector(rstd, "rstd", 1 << DLM_F32, a.N, true))) return st;
  if (!(eps >= 0.f) || std::isinf(eps)) return fail(DLM_ERR_ARG, "eps must be finite and not negative");
  const dlm_tensor* outs[3] = {out, mean, rstd};
  const dlm_tensor* ins[3] = {x, weight, bias};
  if ((st = check_disjoint(outs, 3, ins, 3))) return st;
  if (a.N == 0) return DLM_OK;
  a.x = x->data;
  a.weight = weight->data;
  a.bias = bias ? bias->data : nullptr;
  a.out = out->data;
  a.mean = mean ? static_cast<float*>(mean->data) : nullptr;
  a.rstd = rstd ? static_cast<float*>(rstd->data) : nullptr;
  a.is_bf16 = x->dtype == DLM_BF16;
  a.weight_bf16 = weight->dtype == DLM_BF16;
  a.eps = eps;
  return launch_layer_norm(a, current_stream());
}

size_t dlm_layer_norm_grad_workspace_bytes(int64_t rows, int64_t d) {
  return rows > 0 && d > 0 && d <= kMostNormWidth ? norm_grad_workspace_bytes(rows, d) : 0;
}

int dlm_layer_norm_grad(const dlm_tensor* dout, const dlm_tensor* x, const dlm_tensor* weight, const dlm_tensor* mean,
                        const dlm_tensor* rstd, dlm_tensor* dx, dlm_tensor* dweight, dlm_tensor* dbias, void* workspace,
                        size_t workspace_bytes) {
  clear_error();
  NormArgs a = {};
  int64_t N2, d2;
  int st;
  if ((st = rows_of(x, "x", kMaskBF16F32, &a.N, &a.d, &a.s_x))) return st;
  if ((st = rows_of(dout, "dout", 1 << x->dtype, &N2, &d2, &a.s_dout))) return st;
  if ((st = rows_of(dx, "dx", 1 << x->dtype, &N2, &d2, &a.s_dx))) return st;
  if (!same_shape(x, dout) || !same_shape(x, dx)) return fail(DLM_ERR_SHAPE, "dout and dx must have the shape of x");
  if (a.d < 1 || a.d > kMostNormWidth) return fail(DLM_ERR_SHAPE, "rows must have between 1 and 2^24 elements");
  if ((st = check_vector(weight, "weight", kMaskBF16F32, a.d, false))) return st;
  if ((st = check_vector(mean, "mean", 1 << DLM_F32, a.N, false))) return st;
  if ((st = check_vector(rstd, "rstd", 1 << DLM_F32, a.N, false))) return st;
  if ((st = check_vector(dweight, "dweight", 1 << weight->dtype, a.d, true))) return st;
  if ((st = check_vector(dbias, "dbias", 1 << weight->dtype, a.d, true))) return st;
  const dlm_tensor* outs[3] = {dx, dweight, dbias};
  const dlm_tensor* ins[5] = {dout, x, weight, mean, rstd};
  if ((st = check_disjoint(outs, 3, ins, 5))) return st;
  const dlm_tensor* all[8] = {dout, x, weight, mean, rstd, dx, dweight, dbias};
  if ((dweight || dbias) &&
      (st = check_workspace(workspace, workspace_bytes, dlm_layer_norm_grad_workspace_bytes(a.N, a.d), 16, all, 8)))
    return st;
  if (a.N == 0 && !dweight && !dbias) return DLM_OK;
  a.dout = dout->data;
  a.x = x->data;
  a.weight = weight->data;
  a.mean = static_cast<float*>(mean->data);
  a.rstd = static_cast<float*>(rstd->data);
  a.dx = dx->data;
  a.dweight = dweight ? dweight->data : nullptr;
  a.dbias = dbias ? dbias->data : nullptr;
  a.is_bf16 = x->dtype == DLM_BF16;
  a.weight_bf16 = weight->dtype == DLM_BF16;
  a.workspace = workspace;
  return launch_layer_norm_grad(a, current_stream());
}

size_t dlm_clip_grad_norm_workspace_bytes(void) { return clip_grad_norm_workspace_bytes(); }

int dlm_clip_grad_norm(const dlm_tensor* grads, const dlm_tensor* outs, int32_t count, float max_norm, dlm_tensor* norm,
                       void* workspace, size_t workspace_bytes) {
  clear_error();
  int st;
  if (count < 0 || count > kMaxGradTensors) return fail(DLM_ERR_ARG, "count must be in [0, %d]", kMaxGradTensors);
  if (count > 0 && !grads) return fail(DLM_ERR_NULL, "grads is NULL");
  if (!(max_norm >= 0.f)) return fail(DLM_ERR_ARG, "max_norm must not be negative or NaN");
  if ((st = check_vector(norm, "norm", 1 << DLM_F32, 1, false))) return st;
  if ((st = check_workspace(workspace, workspace_bytes, clip_grad_norm_workspace_bytes(), 8, nullptr, 0))) return st;
  // Nothing thrown leaves a C entry point: the only throwing calls are these vectors'.
  try {
    std::vector<GradTensor> list;
    std::vector<Span> read, written;  // by address, once checked
    list.reserve(count);
    read.reserve(count);
    written.reserve(static_cast<size_t>(count) + 2);
    for (int i = 0; i < count; ++i) {
      const dlm_tensor* g = grads + i;
      const dlm_tensor* o = outs ? outs + i : g;
      constexpr int64_t kMost = int64_t{1} << 40;  // a flat buffer of all gradients is one extent
      if ((st = check_tensor(g, "gradient", kMaskBF16F32, 1, 4, kMost))) return st;
      if (o != g) {
        if ((st = check_tensor(o, "scaled gradient", 1 << g->dtype, 1, 4, kMost))) return st;
        if (!same_shape(g, o)) return fail(DLM_ERR_SHAPE, "tensor %d: the output must have the gradient's shape", i);
      }
      if (numel(g) > kMost) return fail(DLM_ERR_SHAPE, "tensor %d: more than 2^40 elements", i);
      if (!is_dense(g) || !is_dense(o)) return fail(DLM_ERR_STRIDE, "tensor %d must be contiguous", i);
      const int64_t size = numel(g);
      if (size == 0) continue;
      list.push_back({g->data, o->data, size, g->dtype == DLM_BF16});
      const uintptr_t bytes = static_cast<uintptr_t>(size) * elem_size(g->dtype), at = reinterpret_cast<uintptr_t>(g->data);
      const bool in_place = outs && o->data == g->data;
      if (!in_place) read.push_back({at, at + bytes});
      if (outs) {
        const uintptr_t to = reinterpret_cast<uintptr_t>(o->data);
        written.push_back({to, to + bytes});
      }
    }
    const uintptr_t norm_at = reinterpret_cast<uintptr_t>(norm->data), ws_at = reinterpret_cast<uintptr_t>(workspace);
    written.push_back({norm_at, norm_at + sizeof(float)});
    written.push_back({ws_at, ws_at + clip_grad_norm_workspace_bytes()});
    if (!written_apart(&read, &written))
      return fail(DLM_ERR_ARG, "an output overlaps a gradient, another output, norm or the workspace");
    GradArgs a = {};
    a.grads = list.data();
    a.count = static_cast<int>(list.size());
    a.scale = outs != nullptr;
    a.max_norm = max_norm;
    a.norm = static_cast<float*>(norm->data);
    a.workspace = static_cast<double*>(workspace);
    return launch_clip_grad_norm(a, current_stream());
  } catch (const std::bad_alloc&) {
    return fail(DLM_ERR_ARG, "out of host memory for the list of gradients");
  }
}

int dlm_adamw(const dlm_tensor* params, const dlm_tensor* masters, const dlm_tensor* grads, const dlm_tensor* m,
              const dlm_tensor* v, const dlm_tensor* m_scales, const dlm_tensor* v_scales, int32_t count,
              const dlm_adamw_params* hyper) {
  clear_error();
  int st;
  if (count < 0 || count > kMaxGradTensors) return fail(DLM_ERR_ARG, "count must be in [0, %d]", kMaxGradTensors);
  if (count > 0 && (!params || !grads || !m || !v)) return fail(DLM_ERR_NULL, "params, grads, m or v is NULL");
  if ((m_scales == nullptr) != (v_scales == nullptr)) return fail(DLM_ERR_NULL, "m_scales and v_scales must both be given or both be NULL");
  if (!hyper || !hyper->lr || !hyper->step) return fail(DLM_ERR_NULL, "hyper, its lr or its step is NULL");
  const auto in_unit = [](double b) { return b >= 0.0 && b < 1.0; };
  const auto rate = [](double x) { return x >= 0.0 && !std::isinf(x); };
  if (!in_unit(hyper->beta1) || !in_unit(hyper->beta2)) return fail(DLM_ERR_ARG, "beta1 and beta2 must be in [0, 1)");
  if (!rate(hyper->eps) || !rate(hyper->weight_decay)) return fail(DLM_ERR_ARG, "eps and weight_decay must be finite and not negative");
  if (hyper->norm && !(hyper->max_norm >= 0.0)) return fail(DLM_ERR_ARG, "max_norm must not be negative or NaN");
  const uintptr_t scalars[3] = {reinterpret_cast<uintptr_t>(hyper->lr), reinterpret_cast<uintptr_t>(hyper->step),
                                reinterpret_cast<uintptr_t>(hyper->norm)};
  for (const uintptr_t at : scalars)
    if (at % 4 != 0) return fail(DLM_ERR_ALIGN, "lr, step and norm must be 4-byte aligned");
  AdamwArgs a = {};
  a.eight = m_scales != nullptr;
  const int state = a.eight ? 1 << DLM_U8 : 1 << DLM_F32;
  // Nothing thrown leaves a C entry point: the only throwing calls are these vectors'.
  try {
    std::vector<AdamwTensor> list;
    std::vector<Span> read, written;
    list.reserve(count);
    read.reserve(static_cast<size_t>(count) + 3);
    written.reserve(6 * static_cast<size_t>(count));
    for (const uintptr_t at : scalars)
      if (at) read.push_back({at, at + 4});
    for (int i = 0; i < count; ++i) {
      struct Entry {
        const dlm_tensor* t;
        const char* name;
        int mask;
        bool scales;
      };
      const Entry entries[7] = {{grads + i, "gradient", kMaskBF16F32, false},
                                {params + i, "params", masters ? 1 << DLM_BF16 : kMaskBF16F32, false},
                                {masters ? masters + i : nullptr, "masters", 1 << DLM_F32, false},
                                {m + i, "m", state, false},
                                {v + i, "v", state, false},
                                {a.eight ? m_scales + i : nullptr, "m_scales", 1 << DLM_F32, true},
                                {a.eight ? v_scales + i : nullptr, "v_scales", 1 << DLM_F32, true}};
      void* data[7] = {};
      int64_t n = 0;
      for (int k = 0; k < 7; ++k) {
        const Entry& e = entries[k];
        if (!e.t) continue;
        Span span;
        if ((st = list_tensor(e.t, e.name, e.mask, i, &span))) return st;
        if (k == 0) n = numel(e.t);
        if (e.scales ? numel(e.t) != (n + kAdamwBlock - 1) / kAdamwBlock : !same_shape(e.t, grads + i))
          return fail(DLM_ERR_SHAPE, e.scales ? "%s %d: an entry for every 256 elements expected" : "%s %d must have the gradient's shape",
                      e.name, i);
        data[k] = e.t->data;
        if (n > 0) (k == 0 ? read : written).push_back(span);
      }
      if (n == 0) continue;
      list.push_back({data[1], static_cast<float*>(data[2]), data[0], data[3], data[4], static_cast<float*>(data[5]),
                      static_cast<float*>(data[6]), n, params[i].dtype == DLM_BF16, grads[i].dtype == DLM_BF16});
    }
    if (!written_apart(&read, &written)) return fail(DLM_ERR_ARG, "a tensor that is written overlaps another one");
    if (list.empty()) return DLM_OK;
    if ((st = require_error_word())) return st;
    a.tensors = list.data();
    a.count = static_cast<int>(list.size());
    a.beta1 = hyper->beta1;
    a.beta2 = hyper->beta2;
    a.eps = hyper->eps;
    a.weight_decay = hyper->weight_decay;
    a.max_norm = hyper->max_norm;
    a.lr = hyper->lr;
    a.step = hyper->step;
    a.norm = hyper->norm;
    return launch_adamw(a, current_stream());
  } catch (const std::bad_alloc&) {
    return fail(DLM_ERR_ARG, "out of host memory for the list of tensors");
  }
}

}  // extern "C"
