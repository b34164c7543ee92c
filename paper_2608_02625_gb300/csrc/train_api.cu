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

// No output may overlap an input or another output. Null descriptors are skipped.
int check_disjoint(const dlm_tensor* const* outs, int n_outs, const dlm_tensor* const* ins, int n_ins) {
  for (int i = 0; i < n_outs; ++i) {
    if (!outs[i]) continue;
    for (int j = 0; j < n_ins; ++j)
      if (ins[j] && overlaps(outs[i], ins[j])) return fail(DLM_ERR_ARG, "an output overlaps an input");
    for (int j = 0; j < i; ++j)
      if (outs[j] && overlaps(outs[i], outs[j])) return fail(DLM_ERR_ARG, "outputs overlap each other");
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

}  // namespace

extern "C" {

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
  struct Span {
    uintptr_t lo, hi;
  };
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
    // A written range may overlap no other: both lists walked together in the order of their
    // addresses (which tensors allocated one after another often have already).
    const auto before = [](const Span& p, const Span& q) { return p.lo < q.lo; };
    for (std::vector<Span>* v : {&read, &written})
      if (!std::is_sorted(v->begin(), v->end(), before)) std::sort(v->begin(), v->end(), before);
    uintptr_t end = 0, written_end = 0;  // the furthest end so far, of any and of a written range
    for (size_t i = 0, j = 0; i < read.size() || j < written.size();) {
      const bool write = i == read.size() || (j < written.size() && written[j].lo < read[i].lo);
      const Span& p = write ? written[j++] : read[i++];
      if (p.lo < (write ? end : written_end))
        return fail(DLM_ERR_ARG, "an output overlaps a gradient, another output, norm or the workspace");
      end = std::max(end, p.hi);
      if (write) written_end = std::max(written_end, p.hi);
    }
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

}  // extern "C"
