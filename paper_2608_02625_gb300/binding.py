"""Thin Python binding of libdlmrefine (argument marshalling only).

Each function has the name and argument order of its C entry point
(include/dlmrefine.h), takes torch CUDA tensors, builds the dlm_tensor
descriptors, sets the library's stream to torch's current stream of the
tensors' device and calls the library. All computation runs in the CUDA
kernels; a nonzero status raises DlmError. The shared libraries must have been
built (``python -m paper_2608_02625_gb300.build``): there is no fallback.

The compute calls marshal natively (csrc/marshal.cpp) where their arguments are
plain CUDA tensors on the current device; a call with any other argument goes
through ctypes below, which accepts and refuses the same forms.
"""
from __future__ import annotations

import ctypes
import dataclasses
import os

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
library_path = os.path.join(_PKG, "libdlmrefine.so")

DLM_BF16, DLM_F32, DLM_I32, DLM_U8 = 1, 2, 3, 4
_DTYPES = {torch.bfloat16: DLM_BF16, torch.float32: DLM_F32, torch.int32: DLM_I32, torch.uint8: DLM_U8}


class DlmTensor(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("dtype", ctypes.c_int32), ("ndim", ctypes.c_int32),
                ("shape", ctypes.c_int64 * 4), ("stride", ctypes.c_int64 * 4)]


class DlmRefineParams(ctypes.Structure):
    _fields_ = [("edit_threshold", ctypes.c_float), ("remask_k", ctypes.c_int32),
                ("remask_frac", ctypes.c_float), ("mask_id", ctypes.c_int32),
                ("prompt_lens", ctypes.c_void_p), ("seq_lens", ctypes.c_void_p)]


class DlmAdamwParams(ctypes.Structure):
    _fields_ = [("beta1", ctypes.c_double), ("beta2", ctypes.c_double), ("eps", ctypes.c_double),
                ("weight_decay", ctypes.c_double), ("max_norm", ctypes.c_double), ("lr", ctypes.c_void_p),
                ("step", ctypes.c_void_p), ("norm", ctypes.c_void_p)]


class DlmError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"libdlmrefine status {status}: {message}")
        self.status = status


def _load():
    if not os.path.exists(library_path):
        raise ImportError(f"{library_path} is missing: build it with "
                          "`python -m paper_2608_02625_gb300.build` (no CPU fallback exists)")
    lib = ctypes.CDLL(library_path)
    P = ctypes.POINTER(DlmTensor)
    lib.dlm_bidir_attn.argtypes = [P, P, P, P, P]
    lib.dlm_attn_masked.argtypes = [P, P, P, P, P, ctypes.c_int32, ctypes.c_int32, P]
    lib.dlm_vocab_confidence.argtypes = [P, P, P, P]
    lib.dlm_refine_update.argtypes = [P, P, P, P, ctypes.POINTER(DlmRefineParams), P, P, P]
    lib.dlm_refine_step.argtypes = [P, P, P, ctypes.POINTER(DlmRefineParams), P, P, P, P, P, P,
                                    ctypes.c_void_p, ctypes.c_size_t]
    lib.dlm_token_prob.argtypes = [P, P, P, P]
    lib.dlm_lmhead_confidence.argtypes = [P, P, P, P, P, ctypes.c_void_p, ctypes.c_size_t]
    lib.dlm_lmhead_workspace_bytes.argtypes = [ctypes.c_int64]
    lib.dlm_lmhead_workspace_bytes.restype = ctypes.c_size_t
    lib.dlm_lmhead_loss.argtypes = [P] * 5 + [ctypes.c_void_p, ctypes.c_size_t]
    lib.dlm_lmhead_loss_workspace_bytes.argtypes = [ctypes.c_int64, ctypes.c_int64]
    lib.dlm_lmhead_loss_grad.argtypes = [P] * 7 + [ctypes.c_void_p, ctypes.c_size_t]
    lib.dlm_lmhead_loss_grad_workspace_bytes.argtypes = [ctypes.c_int64] * 4
    lib.dlm_layer_norm.argtypes = [P, P, P, ctypes.c_float, P, P, P]
    lib.dlm_layer_norm_grad.argtypes = [P] * 8 + [ctypes.c_void_p, ctypes.c_size_t]
    lib.dlm_layer_norm_grad_workspace_bytes.argtypes = [ctypes.c_int64, ctypes.c_int64]
    lib.dlm_clip_grad_norm.argtypes = [P, P, ctypes.c_int32, ctypes.c_float, P, ctypes.c_void_p, ctypes.c_size_t]
    lib.dlm_clip_grad_norm_workspace_bytes.argtypes = []
    lib.dlm_gated_linear.argtypes = [P] * 3 + [ctypes.c_int32] + [P] * 3
    lib.dlm_gated_linear_grad.argtypes = [P] * 6 + [ctypes.c_int32] + [P] * 4 + [ctypes.c_void_p, ctypes.c_size_t]
    lib.dlm_linear.argtypes = [P] * 3 + [ctypes.c_int32] + [P] * 3 + [ctypes.c_void_p, ctypes.c_size_t]
    lib.dlm_linear_grad.argtypes = [P] * 4 + [ctypes.c_int32] + [P] * 4 + [ctypes.c_void_p, ctypes.c_size_t]
    for f in ("dlm_gated_linear_grad_workspace_bytes", "dlm_linear_workspace_bytes", "dlm_linear_grad_workspace_bytes"):
        getattr(lib, f).argtypes = [ctypes.c_int64] * 3
        getattr(lib, f).restype = ctypes.c_size_t
    lib.dlm_adamw.argtypes = [P] * 7 + [ctypes.c_int32, ctypes.POINTER(DlmAdamwParams)]
    for f in ("dlm_lmhead_loss_workspace_bytes", "dlm_lmhead_loss_grad_workspace_bytes",
              "dlm_layer_norm_grad_workspace_bytes", "dlm_clip_grad_norm_workspace_bytes"):
        getattr(lib, f).restype = ctypes.c_size_t
    lib.dlm_refine_update_ranked.argtypes = [P, P, P, P, P, ctypes.POINTER(DlmRefineParams), P, P, P]
    lib.dlm_refine_step_static.argtypes = [P, P, P, ctypes.POINTER(DlmRefineParams), P, P, P, P, P, P]
    lib.dlm_refine_step_workspace_bytes.argtypes = [ctypes.c_int64]
    lib.dlm_refine_step_workspace_bytes.restype = ctypes.c_size_t
    for f in ("dlm_bidir_attn", "dlm_attn_masked", "dlm_vocab_confidence", "dlm_refine_update", "dlm_refine_step",
              "dlm_refine_step_static", "dlm_token_prob", "dlm_refine_update_ranked", "dlm_lmhead_confidence",
              "dlm_lmhead_loss", "dlm_lmhead_loss_grad", "dlm_layer_norm", "dlm_layer_norm_grad",
              "dlm_clip_grad_norm", "dlm_gated_linear", "dlm_gated_linear_grad", "dlm_linear", "dlm_linear_grad",
              "dlm_adamw", "dlm_set_stream", "dlm_set_attn_tiles_per_unit", "dlm_version",
              "dlm_get_device_error"):
        getattr(lib, f).restype = ctypes.c_int
    lib.dlm_loop_begin.argtypes = [ctypes.c_void_p]
    lib.dlm_loop_end.argtypes = [ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.POINTER(ctypes.c_void_p)]
    lib.dlm_loop_cancel.argtypes = []
    lib.dlm_loop_launch.argtypes = [ctypes.c_void_p]
    lib.dlm_loop_destroy.argtypes = [ctypes.c_void_p]
    for f in ("dlm_loop_begin", "dlm_loop_end", "dlm_loop_cancel", "dlm_loop_launch", "dlm_loop_destroy"):
        getattr(lib, f).restype = ctypes.c_int
    lib.dlm_selftest_wait_timeout.argtypes = [ctypes.c_int64]
    lib.dlm_selftest_wait_timeout.restype = ctypes.c_int
    lib.dlm_set_stream.argtypes = [ctypes.c_void_p]
    lib.dlm_set_attn_tiles_per_unit.argtypes = [ctypes.c_int]
    lib.dlm_get_stream.restype = ctypes.c_void_p
    lib.dlm_status_string.restype = ctypes.c_char_p
    lib.dlm_status_string.argtypes = [ctypes.c_int]
    lib.dlm_last_error.restype = ctypes.c_char_p
    lib.dlm_get_device_error.argtypes = [ctypes.POINTER(ctypes.c_int32), ctypes.c_int]
    return lib


def _load_marshal():
    """The native marshalling, which links against the library loaded above."""
    path = os.path.join(_PKG, "_marshal.so")
    hint = "build it with `python -m paper_2608_02625_gb300.build`"
    if not os.path.exists(path):
        raise ImportError(f"{path} is missing: {hint}")
    try:
        from . import _marshal
    except ImportError as e:
        raise ImportError(f"{path} does not load under this Python and torch ({e}): {hint}") from e
    return _marshal


lib = _load()
_marshal = _load_marshal()


def describe(t: torch.Tensor | None) -> DlmTensor | None:
    """dlm_tensor descriptor of a tensor (no copy)."""
    if t is None:
        return None
    if t.dtype not in _DTYPES:
        raise TypeError(f"unsupported dtype {t.dtype}")
    if t.dim() < 1 or t.dim() > 4:
        raise ValueError("tensors of rank 1..4 only")
    d = DlmTensor()
    n = t.dim()
    d.data = t.data_ptr() if t.numel() else None
    d.dtype = _DTYPES[t.dtype]
    d.ndim = n
    d.shape[:n] = t.shape
    d.stride[:n] = t.stride()
    return d


def _ref(d):
    return ctypes.byref(d) if d is not None else None


def _check(status: int):
    if status != 0:
        msg = lib.dlm_last_error().decode() or lib.dlm_status_string(status).decode()
        raise DlmError(status, msg)


def _done(status) -> bool:
    """Whether the native marshalling took a call (None: it did nothing)."""
    if status is None:
        return False
    _check(status)
    return True


def _prepare(*tensors):
    dev = -1
    for t in tensors:
        if t is None:
            continue
        idx = t.get_device()
        if idx < 0:
            raise ValueError("libdlmrefine takes CUDA tensors")
        if dev < 0:
            dev = idx
        elif idx != dev:
            raise ValueError("all tensors must be on one device")
    if dev < 0:
        raise ValueError("no tensor given")
    if torch.cuda.current_device() != dev:
        torch.cuda.set_device(dev)
    _check(lib.dlm_set_stream(ctypes.c_void_p(torch.cuda.current_stream(dev).cuda_stream)))


def dlm_version() -> int:
    return lib.dlm_version()


def dlm_status_string(status: int) -> str:
    return lib.dlm_status_string(status).decode()


def dlm_bidir_attn(q, k, v, seq_lens, out):
    """Non-causal GQA attention: out[b,i,h] = softmax(q k^T / sqrt(D)) v over keys j < n_b."""
    if _done(_marshal.bidir_attn(q, k, v, seq_lens, out)):
        return out
    _prepare(q, k, v, seq_lens, out)
    dq, dk, dv, ds, do = (describe(t) for t in (q, k, v, seq_lens, out))
    _check(lib.dlm_bidir_attn(_ref(dq), _ref(dk), _ref(dv), _ref(ds), _ref(do)))
    return out


ATTN_FULL, ATTN_BLOCK_CAUSAL, ATTN_BLOCK_LOCAL = 0, 1, 2


def dlm_attn_masked(q, k, v, seq_lens, prompt_lens, mode: int, block: int, out):
    """Attention restricted by a block mask (ATTN_BLOCK_CAUSAL: prompt, earlier
    blocks and the own block; ATTN_BLOCK_LOCAL: prompt and the own block)."""
    if _done(_marshal.attn_masked(q, k, v, seq_lens, prompt_lens, mode, block, out)):
        return out
    _prepare(q, k, v, seq_lens, prompt_lens, out)
    ds = [describe(t) for t in (q, k, v, seq_lens, prompt_lens)]
    do = describe(out)
    _check(lib.dlm_attn_masked(*[_ref(d) for d in ds], int(mode), int(block), _ref(do)))
    return out


def dlm_vocab_confidence(logits, argmax, conf, lse):
    """Per row: argmax (lowest index), max softmax probability, log-sum-exp."""
    if _done(_marshal.vocab_confidence(logits, argmax, conf, lse)):
        return argmax, conf, lse
    _prepare(logits, argmax, conf, lse)
    ds = [describe(t) for t in (logits, argmax, conf, lse)]
    _check(lib.dlm_vocab_confidence(*[_ref(d) for d in ds]))
    return argmax, conf, lse


@dataclasses.dataclass
class RefineParams:
    edit_threshold: float
    remask_k: int
    remask_frac: float
    mask_id: int
    prompt_lens: torch.Tensor  # int32 [B] on the device
    seq_lens: torch.Tensor     # int32 [B] on the device

    def to_c(self) -> DlmRefineParams:
        for t in (self.prompt_lens, self.seq_lens):
            if t.dtype != torch.int32 or not t.is_cuda or not t.is_contiguous():
                raise ValueError("prompt_lens / seq_lens must be contiguous int32 CUDA tensors")
        return DlmRefineParams(float(self.edit_threshold), int(self.remask_k), float(self.remask_frac),
                               int(self.mask_id), self.prompt_lens.data_ptr(), self.seq_lens.data_ptr())


_marshal.set_params_type(RefineParams)


def dlm_refine_update(tokens, mask, argmax, conf, params: RefineParams, new_tokens, new_mask, n_edits):
    """Commit masked positions, edit confident changes, remask the k least confident."""
    if _done(_marshal.refine_update(tokens, mask, argmax, conf, params, new_tokens, new_mask, n_edits)):
        return new_tokens, new_mask, n_edits
    _prepare(tokens, mask, argmax, conf, new_tokens, new_mask, n_edits, params.prompt_lens, params.seq_lens)
    ds = [describe(t) for t in (tokens, mask, argmax, conf)]
    outs = [describe(t) for t in (new_tokens, new_mask, n_edits)]
    cp = params.to_c()
    _check(lib.dlm_refine_update(*[_ref(d) for d in ds], ctypes.byref(cp), *[_ref(d) for d in outs]))
    return new_tokens, new_mask, n_edits


def dlm_lmhead_workspace_bytes(rows: int) -> int:
    return lib.dlm_lmhead_workspace_bytes(int(rows))


def dlm_lmhead_confidence(hidden, weight, argmax, conf, lse, workspace):
    """argmax / conf / lse of hidden @ weight^T per row, without materialising the logits."""
    if _done(_marshal.lmhead_confidence(hidden, weight, argmax, conf, lse, workspace)):
        return argmax, conf, lse
    _prepare(hidden, weight, argmax, conf, lse, workspace)
    if not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous")
    ds = [describe(t) for t in (hidden, weight, argmax, conf, lse)]
    nbytes = workspace.numel() * workspace.element_size()
    _check(lib.dlm_lmhead_confidence(*[_ref(d) for d in ds], ctypes.c_void_p(workspace.data_ptr() if nbytes else None),
                                     ctypes.c_size_t(nbytes)))
    return argmax, conf, lse


def _workspace(workspace):
    """(address, bytes) of a workspace tensor; (None, 0) for None."""
    if workspace is None:
        return ctypes.c_void_p(None), ctypes.c_size_t(0)
    if not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous")
    nbytes = workspace.numel() * workspace.element_size()
    return ctypes.c_void_p(workspace.data_ptr() if nbytes else None), ctypes.c_size_t(nbytes)


def dlm_lmhead_loss_workspace_bytes(rows: int, d: int) -> int:
    return lib.dlm_lmhead_loss_workspace_bytes(int(rows), int(d))


def dlm_lmhead_loss(hidden, weight, targets, loss, lse, workspace):
    """loss / lse per row: the cross entropy of targets under hidden @ weight^T, without
    materialising the logits; 0 for rows whose target is outside [0, V)."""
    if _done(_marshal.lmhead_loss(hidden, weight, targets, loss, lse, workspace)):
        return loss, lse
    _prepare(hidden, weight, targets, loss, lse, workspace)
    ds = [describe(t) for t in (hidden, weight, targets, loss, lse)]
    _check(lib.dlm_lmhead_loss(*[_ref(d) for d in ds], *_workspace(workspace)))
    return loss, lse


def dlm_lmhead_loss_grad_workspace_bytes(rows: int, vocab: int, d: int, piece: int = 0) -> int:
    """Bytes that let dlm_lmhead_loss_grad take `piece` columns of the vocabulary at a time
    (0: about 2 GB of them)."""
    return lib.dlm_lmhead_loss_grad_workspace_bytes(int(rows), int(vocab), int(d), int(piece))


def dlm_lmhead_loss_grad(hidden, weight, targets, lse, dloss, d_hidden, d_weight, workspace):
    """Gradients of sum(dloss * loss) of dlm_lmhead_loss; d_hidden or d_weight may be None."""
    if _done(_marshal.lmhead_loss_grad(hidden, weight, targets, lse, dloss, d_hidden, d_weight, workspace)):
        return d_hidden, d_weight
    _prepare(hidden, weight, targets, lse, dloss, d_hidden, d_weight, workspace)
    ds = [describe(t) for t in (hidden, weight, targets, lse, dloss, d_hidden, d_weight)]
    _check(lib.dlm_lmhead_loss_grad(*[_ref(d) for d in ds], *_workspace(workspace)))
    return d_hidden, d_weight


def dlm_layer_norm(x, weight, bias, eps: float, out, mean, rstd):
    """out = (x - mean) * rstd * weight + bias over the last dimension. bias, mean
    and rstd may be None (mean and rstd are what dlm_layer_norm_grad reads)."""
    if _done(_marshal.layer_norm(x, weight, bias, eps, out, mean, rstd)):
        return out, mean, rstd
    _prepare(x, weight, bias, out, mean, rstd)
    dx, dw, db, do, dm, dr = (describe(t) for t in (x, weight, bias, out, mean, rstd))
    _check(lib.dlm_layer_norm(_ref(dx), _ref(dw), _ref(db), float(eps), _ref(do), _ref(dm), _ref(dr)))
    return out, mean, rstd


def dlm_layer_norm_grad_workspace_bytes(rows: int, d: int) -> int:
    return lib.dlm_layer_norm_grad_workspace_bytes(int(rows), int(d))


def dlm_layer_norm_grad(dout, x, weight, mean, rstd, dx, dweight, dbias, workspace):
    """Gradients of dlm_layer_norm. dweight and dbias may be None; the workspace too
    where both are."""
    if _done(_marshal.layer_norm_grad(dout, x, weight, mean, rstd, dx, dweight, dbias, workspace)):
        return dx, dweight, dbias
    _prepare(dout, x, weight, mean, rstd, dx, dweight, dbias, workspace)
    ds = [describe(t) for t in (dout, x, weight, mean, rstd, dx, dweight, dbias)]
    _check(lib.dlm_layer_norm_grad(*[_ref(d) for d in ds], *_workspace(workspace)))
    return dx, dweight, dbias


def dlm_clip_grad_norm_workspace_bytes() -> int:
    return lib.dlm_clip_grad_norm_workspace_bytes()


def dlm_clip_grad_norm(grads, outs, max_norm: float, norm, workspace):
    """norm: over every element of every tensor of `grads`; outs[i] = grads[i] scaled so
    that the norm is at most max_norm (outs may be grads: in place; None: the norm alone)."""
    if _done(_marshal.clip_grad_norm(grads, outs, max_norm, norm, workspace)):
        return outs, norm
    if outs is not None and len(outs) != len(grads):
        raise ValueError("outs must have one tensor per gradient")
    _prepare(norm, workspace, *grads, *(outs or ()))
    n = len(grads)
    dg = (DlmTensor * max(1, n))(*[describe(t) for t in grads])
    do = None if outs is None else (DlmTensor * max(1, n))(*[describe(t) for t in outs])
    dn = describe(norm)
    _check(lib.dlm_clip_grad_norm(dg, do, n, float(max_norm), _ref(dn), *_workspace(workspace)))
    return outs, norm


ACT_NONE, ACT_SILU, ACT_GELU = 0, 1, 2  # GELU in its tanh form


def dlm_gated_linear(x, w_gate, w_up, act: int, out, gate, up):
    """out = act(x @ w_gate^T) * (x @ w_up^T), the first half of a gated feed-forward block.
    gate and up (the two products, which dlm_gated_linear_grad reads) may both be None."""
    if _done(_marshal.gated_linear(x, w_gate, w_up, act, out, gate, up)):
        return out, gate, up
    _prepare(x, w_gate, w_up, out, gate, up)
    ds = [describe(t) for t in (x, w_gate, w_up, out, gate, up)]
    _check(lib.dlm_gated_linear(*[_ref(d) for d in ds[:3]], int(act), *[_ref(d) for d in ds[3:]]))
    return out, gate, up


def dlm_gated_linear_grad_workspace_bytes(rows: int, f: int, d: int) -> int:
    return lib.dlm_gated_linear_grad_workspace_bytes(int(rows), int(f), int(d))


def dlm_gated_linear_grad(dout, x, w_gate, w_up, gate, up, act: int, add, dx, dw_gate, dw_up, workspace):
    """Gradients of dlm_gated_linear. add (what else goes to dx; may be dx itself), dx, and
    dw_gate with dw_up may be None."""
    if _done(_marshal.gated_linear_grad(dout, x, w_gate, w_up, gate, up, act, add, dx, dw_gate, dw_up, workspace)):
        return dx, dw_gate, dw_up
    _prepare(dout, x, w_gate, w_up, gate, up, add, dx, dw_gate, dw_up, workspace)
    ds = [describe(t) for t in (dout, x, w_gate, w_up, gate, up, add, dx, dw_gate, dw_up)]
    _check(lib.dlm_gated_linear_grad(*[_ref(d) for d in ds[:6]], int(act), *[_ref(d) for d in ds[6:]], *_workspace(workspace)))
    return dx, dw_gate, dw_up


def dlm_linear_workspace_bytes(rows: int, m: int, k: int) -> int:
    return lib.dlm_linear_workspace_bytes(int(rows), int(m), int(k))


def dlm_linear(x, weight, bias, act: int, residual, out, pre, workspace):
    """out = act(x @ weight^T + bias) + residual. bias, residual (may be out itself), pre (the
    activation's argument, which dlm_linear_grad reads) may be None; the workspace too where
    dlm_linear_workspace_bytes is 0."""
    if _done(_marshal.linear(x, weight, bias, act, residual, out, pre, workspace)):
        return out, pre
    _prepare(x, weight, bias, residual, out, pre, workspace)
    ds = [describe(t) for t in (x, weight, bias, residual, out, pre)]
    _check(lib.dlm_linear(*[_ref(d) for d in ds[:3]], int(act), *[_ref(d) for d in ds[3:]], *_workspace(workspace)))
    return out, pre


def dlm_linear_grad_workspace_bytes(rows: int, m: int, k: int) -> int:
    return lib.dlm_linear_grad_workspace_bytes(int(rows), int(m), int(k))


def dlm_linear_grad(dout, x, weight, pre, act: int, add, dx, dweight, dbias, workspace):
    """Gradients of dlm_linear. pre is None with ACT_NONE; add (what else goes to dx; may be dx
    itself), dx, dweight and dbias may be None."""
    if _done(_marshal.linear_grad(dout, x, weight, pre, act, add, dx, dweight, dbias, workspace)):
        return dx, dweight, dbias
    _prepare(dout, x, weight, pre, add, dx, dweight, dbias, workspace)
    ds = [describe(t) for t in (dout, x, weight, pre, add, dx, dweight, dbias)]
    _check(lib.dlm_linear_grad(*[_ref(d) for d in ds[:4]], int(act), *[_ref(d) for d in ds[4:]], *_workspace(workspace)))
    return dx, dweight, dbias


@dataclasses.dataclass
class AdamwParams:
    lr: torch.Tensor           # float32 [1] on the device
    step: torch.Tensor         # int32 [1] on the device: the number of the step, from 1 on
    beta1: float = 0.9
    beta2: float = 0.999
    eps: float = 1e-8
    weight_decay: float = 0.0
    norm: torch.Tensor | None = None  # float32 [1] on the device: gradients are clipped by it
    max_norm: float = float("inf")

    def to_c(self) -> DlmAdamwParams:
        for name, dtype in (("lr", torch.float32), ("step", torch.int32), ("norm", torch.float32)):
            t = getattr(self, name)
            if t is None and name == "norm":
                continue
            if t is None or t.dtype != dtype or not t.is_cuda or t.numel() != 1:
                raise ValueError("lr, step and norm must be one-element CUDA tensors (float32, int32, float32)")
        return DlmAdamwParams(float(self.beta1), float(self.beta2), float(self.eps), float(self.weight_decay),
                              float(self.max_norm), self.lr.data_ptr(), self.step.data_ptr(),
                              None if self.norm is None else self.norm.data_ptr())


_marshal.set_adamw_type(AdamwParams)

ADAMW_BLOCK = 256  # elements that share a scale where states are held in 8 bits


def dlm_adamw(params, masters, grads, m, v, m_scales, v_scales, hyper: AdamwParams):
    """One AdamW step over lists of tensors, in place: params (with masters, float32 tensors
    that hold the weights, their bfloat16 copies), m and v. m_scales and v_scales None: m and
    v are float32; else uint8 codes (e4m3, of sqrt(v) for v) with a float32 scale for every
    ADAMW_BLOCK elements. All states are zeros before the first step."""
    if _done(_marshal.adamw(params, masters, grads, m, v, m_scales, v_scales, hyper)):
        return params
    lists = [params, masters, grads, m, v, m_scales, v_scales]
    if any(x is not None and len(x) != len(params) for x in lists):
        raise ValueError("every list must have one tensor per parameter")
    _prepare(hyper.lr, hyper.step, hyper.norm, *[t for x in lists if x is not None for t in x])
    n = len(params)
    ds = [None if x is None else (DlmTensor * max(1, n))(*[describe(t) for t in x]) for x in lists]
    cp = hyper.to_c()
    _check(lib.dlm_adamw(*ds, n, ctypes.byref(cp)))
    return params


def dlm_token_prob(logits, tokens, lse, prob):
    """prob[r] = exp(logits[r, tokens[r]] - lse[r]) (0 for a token outside [0, V))."""
    if _done(_marshal.token_prob(logits, tokens, lse, prob)):
        return prob
    _prepare(logits, tokens, lse, prob)
    ds = [describe(t) for t in (logits, tokens, lse, prob)]
    _check(lib.dlm_token_prob(*[_ref(d) for d in ds]))
    return prob


def dlm_refine_update_ranked(tokens, mask, argmax, conf, tok_prob, params: RefineParams, new_tokens, new_mask,
                             n_edits):
    """dlm_refine_update remasking by the probability of each position's resulting token."""
    if _done(_marshal.refine_update_ranked(tokens, mask, argmax, conf, tok_prob, params, new_tokens,
                                           new_mask, n_edits)):
        return new_tokens, new_mask, n_edits
    _prepare(tokens, mask, argmax, conf, tok_prob, new_tokens, new_mask, n_edits, params.prompt_lens,
             params.seq_lens)
    ds = [describe(t) for t in (tokens, mask, argmax, conf, tok_prob)]
    outs = [describe(t) for t in (new_tokens, new_mask, n_edits)]
    cp = params.to_c()
    _check(lib.dlm_refine_update_ranked(*[_ref(d) for d in ds], ctypes.byref(cp), *[_ref(d) for d in outs]))
    return new_tokens, new_mask, n_edits


def dlm_refine_step_workspace_bytes(batch: int) -> int:
    return lib.dlm_refine_step_workspace_bytes(int(batch))


def dlm_refine_step(logits, tokens, mask, params: RefineParams, argmax, conf, lse, new_tokens, new_mask, n_edits,
                    workspace):
    """Vocabulary reduction and refine update in one call.

    workspace: a CUDA tensor of at least dlm_refine_step_workspace_bytes(B) bytes,
    zero before its first use and, untouched by the present implementation, after
    each call."""
    if _done(_marshal.refine_step(logits, tokens, mask, params, argmax, conf, lse, new_tokens, new_mask,
                                  n_edits, workspace)):
        return argmax, conf, lse, new_tokens, new_mask, n_edits
    _prepare(logits, tokens, mask, argmax, conf, lse, new_tokens, new_mask, n_edits, workspace,
             params.prompt_lens, params.seq_lens)
    if not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous")
    ins = [describe(t) for t in (logits, tokens, mask)]
    outs = [describe(t) for t in (argmax, conf, lse, new_tokens, new_mask, n_edits)]
    cp = params.to_c()
    nbytes = workspace.numel() * workspace.element_size()
    _check(lib.dlm_refine_step(*[_ref(d) for d in ins], ctypes.byref(cp), *[_ref(d) for d in outs],
                               ctypes.c_void_p(workspace.data_ptr() if nbytes else None), ctypes.c_size_t(nbytes)))
    return argmax, conf, lse, new_tokens, new_mask, n_edits


def dlm_refine_step_static(logits, tokens, mask, params: RefineParams, argmax, conf, lse, new_tokens, new_mask,
                           n_edits):
    """dlm_refine_step without a workspace, for callers that cannot allocate
    device memory. The first call on a device sets that device up (make it
    before any stream capture)."""
    if _done(_marshal.refine_step_static(logits, tokens, mask, params, argmax, conf, lse, new_tokens,
                                         new_mask, n_edits)):
        return argmax, conf, lse, new_tokens, new_mask, n_edits
    _prepare(logits, tokens, mask, argmax, conf, lse, new_tokens, new_mask, n_edits, params.prompt_lens,
             params.seq_lens)
    ins = [describe(t) for t in (logits, tokens, mask)]
    outs = [describe(t) for t in (argmax, conf, lse, new_tokens, new_mask, n_edits)]
    cp = params.to_c()
    _check(lib.dlm_refine_step_static(*[_ref(d) for d in ins], ctypes.byref(cp), *[_ref(d) for d in outs]))
    return argmax, conf, lse, new_tokens, new_mask, n_edits


class RefineLoop:
    """A recorded refine pass that the GPU repeats until no confident edit
    remains or max_steps passes have run (one graph launch)."""

    def __init__(self, handle: int, device: torch.device, steps_out: torch.Tensor):
        self._h = handle
        self.device = device
        self.steps_out = steps_out

    def launch(self):
        """Runs the loop on the current stream of its device; steps_out then
        holds the number of passes once the stream reaches that point."""
        if not self._h:
            raise ValueError("the loop has been destroyed")
        if _done(_marshal.loop_launch(self._h, self.device.index)):
            return
        torch.cuda.set_device(self.device)
        _check(lib.dlm_set_stream(ctypes.c_void_p(torch.cuda.current_stream(self.device).cuda_stream)))
        _check(lib.dlm_loop_launch(ctypes.c_void_p(self._h)))

    def close(self):
        if self._h:
            _check(lib.dlm_loop_destroy(ctypes.c_void_p(self._h)))
            self._h = None


def dlm_loop_begin(steps_out: torch.Tensor):
    """Starts recording one refine pass on the current (non-default) stream."""
    if steps_out.dtype != torch.int32 or steps_out.numel() != 1:
        raise ValueError("steps_out must be a one-element int32 CUDA tensor")
    _prepare(steps_out)
    _check(lib.dlm_loop_begin(ctypes.c_void_p(steps_out.data_ptr())))


def dlm_loop_end(n_edits: torch.Tensor, max_steps: int, steps_out: torch.Tensor) -> RefineLoop:
    """Ends the recording: the pass repeats while passes < max_steps and some
    n_edits[b] > 0."""
    if n_edits.dtype != torch.int32 or not n_edits.is_contiguous() or n_edits.dim() != 1:
        lib.dlm_loop_cancel()
        raise ValueError("n_edits must be a contiguous int32 [B] CUDA tensor")
    h = ctypes.c_void_p()
    _check(lib.dlm_loop_end(ctypes.c_void_p(n_edits.data_ptr() if n_edits.numel() else None), n_edits.numel(),
                            int(max_steps), ctypes.byref(h)))
    return RefineLoop(h.value, n_edits.device, steps_out)


def dlm_loop_cancel():
    """Ends an unfinished recording on this thread, keeping nothing."""
    _check(lib.dlm_loop_cancel())


def dlm_set_attn_tiles_per_unit(tiles: int):
    """Query tiles per attention work unit on this thread: 0 automatic, 1 or 2."""
    _check(lib.dlm_set_attn_tiles_per_unit(int(tiles)))


def dlm_selftest_wait_timeout(budget_ns: int, device: int | None = None):
    """Runs a kernel whose bounded wait on a barrier nothing arrives on gives
    up after budget_ns; afterwards device_error() holds DLM_DEVERR_TIMEOUT."""
    dev = torch.cuda.current_device() if device is None else device
    torch.cuda.set_device(dev)
    _check(lib.dlm_set_stream(ctypes.c_void_p(torch.cuda.current_stream(dev).cuda_stream)))
    _check(lib.dlm_selftest_wait_timeout(int(budget_ns)))


def device_error(clear: bool = True) -> int:
    """The device error word (DLM_DEVERR_* bits) of the current device; synchronises."""
    bits = ctypes.c_int32(0)
    _check(lib.dlm_get_device_error(ctypes.byref(bits), 1 if clear else 0))
    return bits.value
