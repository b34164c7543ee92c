"""Host-side validation of the entry points of training the refiner's last layer:
what is refused, with nothing launched (fake device pointers, never read)."""
import ctypes

import pytest

from test_abi import BF16, F32, I32, MB, T, U8, built  # noqa: F401


def call(name, *args):
    from paper_2608_02625_gb300.binding import DlmTensor, lib
    return getattr(lib, name)(*(ctypes.byref(a) if isinstance(a, DlmTensor) else a for a in args))


def norm_args(N=6, d=64, dt=BF16, wdt=F32):
    return dict(x=T(dt, [N, d], 1 * MB), w=T(wdt, [d], 2 * MB), b=T(wdt, [d], 3 * MB), eps=1e-5, out=T(dt, [N, d], 4 * MB),
                mean=T(F32, [N], 5 * MB), rstd=T(F32, [N], 6 * MB))


NORM = {
    "null_x": (dict(x=None), -1), "null_weight": (dict(w=None), -1), "null_out": (dict(out=None), -1),
    "x_int": (dict(x=T(I32, [6, 64], MB)), -2), "out_dtype": (dict(out=T(F32, [6, 64], 4 * MB)), -2),
    "bias_dtype": (dict(b=T(BF16, [64], 3 * MB)), -2), "mean_dtype": (dict(mean=T(BF16, [6], 5 * MB)), -2),
    "rank_1": (dict(x=T(BF16, [64], MB)), -3), "out_shape": (dict(out=T(BF16, [6, 63], 4 * MB)), -3),
    "weight_length": (dict(w=T(F32, [63], 2 * MB)), -3), "rstd_length": (dict(rstd=T(F32, [5], 6 * MB)), -3),
    "no_columns": (dict(x=T(BF16, [6, 0], MB), out=T(BF16, [6, 0], 4 * MB), w=T(F32, [0], 2 * MB)), -3),
    "too_wide": (dict(x=T(BF16, [1, 2 ** 24 + 8], MB), out=T(BF16, [1, 2 ** 24 + 8], 4 * MB)), -3),
    "columns_apart": (dict(x=T(BF16, [6, 64], MB, [128, 2])), -4), "rows_overlap": (dict(x=T(BF16, [6, 64], MB, [32, 1])), -4),
    "uneven_rows": (dict(x=T(BF16, [2, 3, 64], MB, [1000, 64, 1]), out=T(BF16, [2, 3, 64], 4 * MB)), -4),
    "weight_apart": (dict(w=T(F32, [64], 2 * MB, [2])), -4), "mean_misaligned": (dict(mean=T(F32, [6], 5 * MB + 2)), -5),
    "eps_negative": (dict(eps=-1e-5), -6), "eps_nan": (dict(eps=float("nan")), -6), "eps_inf": (dict(eps=float("inf")), -6),
    "in_place": (dict(out=T(BF16, [6, 64], MB)), -6), "out_on_weight": (dict(out=T(BF16, [6, 64], 2 * MB + 16)), -6),
    "mean_on_rstd": (dict(mean=T(F32, [6], 6 * MB + 8)), -6),
}


@pytest.mark.parametrize("case", NORM)
def test_layer_norm_refuses(case):
    over, status = NORM[case]
    a = {**norm_args(), **over}
    assert call("dlm_layer_norm", *a.values()) == status


def grad_args(N=6, d=64, dt=BF16, wdt=F32):
    return dict(dout=T(dt, [N, d], 1 * MB), x=T(dt, [N, d], 2 * MB), w=T(wdt, [d], 3 * MB), mean=T(F32, [N], 4 * MB),
                rstd=T(F32, [N], 5 * MB), dx=T(dt, [N, d], 6 * MB), dw=T(wdt, [d], 7 * MB), db=T(wdt, [d], 8 * MB),
                ws=ctypes.c_void_p(9 * MB), nbytes=ctypes.c_size_t(1 << 20))


GRAD = {
    "null_dout": (dict(dout=None), -1), "null_mean": (dict(mean=None), -1), "null_dx": (dict(dx=None), -1),
    "null_workspace": (dict(ws=None), -1), "dout_dtype": (dict(dout=T(F32, [6, 64], MB)), -2),
    "dweight_dtype": (dict(dw=T(BF16, [64], 7 * MB)), -2), "dx_shape": (dict(dx=T(BF16, [5, 64], 6 * MB)), -3),
    "dbias_length": (dict(db=T(F32, [65], 8 * MB)), -3), "dout_broadcast": (dict(dout=T(BF16, [6, 64], MB, [0, 0])), -4),
    "rows_broadcast": (dict(dout=T(BF16, [6, 64], MB, [0, 1])), -4),
    "workspace_misaligned": (dict(ws=ctypes.c_void_p(9 * MB + 8)), -5),
    "workspace_small": (dict(nbytes=ctypes.c_size_t(6 * 2 * 64 * 4 - 1)), -6),
    "dx_on_dout": (dict(dx=T(BF16, [6, 64], MB)), -6), "dw_on_db": (dict(dw=T(F32, [64], 8 * MB + 4)), -6),
    "workspace_on_x": (dict(ws=ctypes.c_void_p(2 * MB)), -6),
}


@pytest.mark.parametrize("case", GRAD)
def test_layer_norm_grad_refuses(case):
    over, status = GRAD[case]
    a = {**grad_args(), **over}
    assert call("dlm_layer_norm_grad", *a.values()) == status


def clip(grads, outs, max_norm=1.0, norm=None, ws=200 * MB, nbytes=1 << 20, count=None):
    from paper_2608_02625_gb300.binding import DlmTensor, lib
    arr = lambda ts: None if ts is None else (DlmTensor * max(1, len(ts)))(*ts)  # noqa: E731
    norm = T(F32, [1], 100 * MB) if norm is None else norm
    return lib.dlm_clip_grad_norm(arr(grads), arr(outs), len(grads or []) if count is None else count, max_norm,
                                  ctypes.byref(norm), ctypes.c_void_p(ws), nbytes)


def test_clip_refuses():
    g = [T(BF16, [100], 1 * MB), T(F32, [7, 3], 2 * MB)]
    o = [T(BF16, [100], 3 * MB), T(F32, [7, 3], 4 * MB)]
    assert clip(None, None, count=2) == -1
    assert clip(g, o, ws=None) == -1
    assert clip(g, o, norm=T(F32, [2], 100 * MB)) == -3
    assert clip(g, o, norm=T(BF16, [1], 100 * MB)) == -2
    assert clip(g, o, ws=200 * MB + 4) == -5
    assert clip(g, o, nbytes=100) == -6
    assert clip(g, o, max_norm=-1.0) == -6
    assert clip(g, o, max_norm=float("nan")) == -6
    assert clip(g, o, count=-1) == -6
    assert clip(g, o, count=20000) == -6
    assert clip([T(I32, [4], MB)], None) == -2
    assert clip([g[0], T(F32, [7, 3], 2 * MB, [4, 1])], None) == -4           # not contiguous
    assert clip(g, [T(F32, [100], 3 * MB), o[1]]) == -2
    assert clip(g, [T(BF16, [99], 3 * MB), o[1]]) == -3
    assert clip(g, [o[0], T(F32, [7, 3], 4 * MB, [4, 1])]) == -4
    assert clip([T(F32, [2 ** 31 - 1, 2 ** 10], MB)], None) == -3              # more than 2^40 elements
    # overlaps of what is written: a tensor twice in place, an output on another gradient,
    # on its own one but not exactly, on norm, on the workspace
    assert clip([g[0], g[0]], [g[0], g[0]]) == -6
    assert clip(g, [o[0], T(F32, [7, 3], 1 * MB + 16)]) == -6
    assert clip(g, [T(BF16, [100], 1 * MB + 2), o[1]]) == -6
    assert clip(g, [o[0], o[0]]) == -2
    assert clip([g[0], g[0]], [o[0], o[0]]) == -6
    assert clip(g, [T(BF16, [100], 100 * MB - 100), o[1]]) == -6
    assert clip(g, [T(BF16, [100], 200 * MB + 100), o[1]]) == -6
    assert clip([T(F32, [30], 100 * MB - 60)], None) == -6                     # norm on a gradient


def test_workspace_sizes():
    from paper_2608_02625_gb300 import binding as B
    assert B.dlm_layer_norm_grad_workspace_bytes(0, 64) == 0
    assert B.dlm_layer_norm_grad_workspace_bytes(6, 64) == 6 * 2 * 64 * 4
    assert B.dlm_layer_norm_grad_workspace_bytes(10 ** 6, 64) == B.dlm_layer_norm_grad_workspace_bytes(10 ** 7, 64)
    assert B.dlm_layer_norm_grad_workspace_bytes(10 ** 6, 2 ** 24) > 0
    assert B.dlm_layer_norm_grad_workspace_bytes(6, 2 ** 24 + 1) == B.dlm_layer_norm_grad_workspace_bytes(6, 2 ** 62) == 0
    assert B.dlm_clip_grad_norm_workspace_bytes() > 0


def loss_args(N=6, V=50, d=64):
    return dict(h=T(BF16, [N, d], 1 * MB), w=T(BF16, [V, d], 2 * MB), t=T(I32, [N], 3 * MB), loss=T(F32, [N], 4 * MB),
                lse=T(F32, [N], 5 * MB), ws=ctypes.c_void_p(6 * MB), nbytes=ctypes.c_size_t(1 << 24))


SHARED = {
    "null_hidden": (dict(h=None), -1), "null_weight": (dict(w=None), -1), "null_targets": (dict(t=None), -1),
    "null_lse": (dict(lse=None), -1), "null_workspace": (dict(ws=None), -1),
    "hidden_f32": (dict(h=T(F32, [6, 64], MB)), -2), "weight_f32": (dict(w=T(F32, [50, 64], 2 * MB)), -2),
    "targets_u8": (dict(t=T(U8, [6], 3 * MB)), -2), "lse_bf16": (dict(lse=T(BF16, [6], 5 * MB)), -2),
    "width": (dict(w=T(BF16, [50, 72], 2 * MB)), -3), "targets_length": (dict(t=T(I32, [5], 3 * MB)), -3),
    "no_vocabulary": (dict(w=T(BF16, [0, 64], 2 * MB)), -3),
    "width_not_8": (dict(h=T(BF16, [6, 60], MB), w=T(BF16, [50, 60], 2 * MB, [64, 1])), -3),
    "hidden_apart": (dict(h=T(BF16, [6, 64], MB, [128, 2])), -4), "weight_overlap": (dict(w=T(BF16, [50, 64], 2 * MB, [8, 1])), -4),
    "targets_apart": (dict(t=T(I32, [6], 3 * MB, [2])), -4), "weight_base": (dict(w=T(BF16, [50, 64], 2 * MB + 2)), -5),
    "weight_stride": (dict(w=T(BF16, [50, 64], 2 * MB, [65, 1])), -5), "workspace_misaligned": (dict(ws=ctypes.c_void_p(6 * MB + 8)), -5),
    "workspace_small": (dict(nbytes=ctypes.c_size_t(1000)), -6), "workspace_on_weight": (dict(ws=ctypes.c_void_p(2 * MB)), -6),
}
LOSS = {
    "loss_on_lse": (dict(loss=T(F32, [6], 5 * MB + 4)), -6), "loss_on_hidden": (dict(loss=T(F32, [6], 1 * MB + 16)), -6),
    "loss_on_targets": (dict(loss=T(F32, [6], 3 * MB)), -6), "loss_length": (dict(loss=T(F32, [7], 4 * MB)), -3),
}


@pytest.mark.parametrize("case", [*SHARED, *LOSS])
def test_loss_refuses(case):
    over, status = {**SHARED, **LOSS}[case]
    assert call("dlm_lmhead_loss", *{**loss_args(), **over}.values()) == status


def loss_grad_args(N=6, V=50, d=64):
    a = loss_args(N, V, d)
    return dict(h=a["h"], w=a["w"], t=a["t"], lse=a["lse"], dloss=T(F32, [N], 4 * MB), dh=T(BF16, [N, d], 10 * MB),
                dw=T(BF16, [V, d], 11 * MB), ws=a["ws"], nbytes=a["nbytes"])


LOSS_GRAD = {
    "null_dloss": (dict(dloss=None), -1), "no_gradient": (dict(dh=None, dw=None), -1),
    "dh_f32": (dict(dh=T(F32, [6, 64], 10 * MB)), -2), "dw_f32": (dict(dw=T(F32, [50, 64], 11 * MB)), -2),
    "dh_shape": (dict(dh=T(BF16, [2, 3, 64], 10 * MB)), -3), "dw_shape": (dict(dw=T(BF16, [49, 64], 11 * MB)), -3),
    "dh_rows_overlap": (dict(dh=T(BF16, [6, 64], 10 * MB, [32, 1])), -4), "dw_base": (dict(dw=T(BF16, [50, 64], 11 * MB + 8)), -5),
    "dw_rows_overlap": (dict(dw=T(BF16, [50, 64], 11 * MB, [56, 1])), -4), "dh_on_hidden": (dict(dh=T(BF16, [6, 64], MB)), -6),
    "dw_on_weight": (dict(dw=T(BF16, [50, 64], 2 * MB)), -6), "dw_on_dh": (dict(dw=T(BF16, [50, 64], 10 * MB)), -6),
    "workspace_on_dw": (dict(ws=ctypes.c_void_p(11 * MB)), -6),
}


@pytest.mark.parametrize("case", [*SHARED, *LOSS_GRAD])
def test_loss_grad_refuses(case):
    over, status = {**SHARED, **LOSS_GRAD}[case]
    assert call("dlm_lmhead_loss_grad", *{**loss_grad_args(), **over}.values()) == status


def test_loss_workspace_sizes():
    from paper_2608_02625_gb300 import binding as B
    assert B.dlm_lmhead_loss_workspace_bytes(0, 64) == B.dlm_lmhead_loss_workspace_bytes(5, 0) == 0
    size = B.dlm_lmhead_loss_grad_workspace_bytes
    assert size(0, 10, 64) == size(5, 0, 64) == size(5, 10, 64, -1) == 0
    assert size(256, 10 ** 5, 64, 512) - size(256, 10 ** 5, 64, 256) == 256 * 256 * 2
    assert size(128, 10 ** 5, 64, 257) == size(128, 10 ** 5, 64, 512)
    assert size(128, 300, 64, 10 ** 6) == size(128, 300, 64, 300)
    assert size(16384, 151552, 2048) < 3 * 2 ** 30
    assert size(128, 300, 64, 2 ** 63 - 1) == size(128, 300, 64, 300)


@pytest.mark.parametrize("stride,status", [(2 ** 39, -4), (2 ** 60, -4), (2 ** 62 + 8, -4), (2 ** 39 - 8, None)])
def test_rows_further_apart_than_a_copy_can_address(stride, status):
    """2^40 bytes from row to row are refused before anything else of the device is asked for;
    a stride below passes (to the check of the workspace, too small here)."""
    far = lambda at: T(BF16, [2, 64], at, [stride, 1])  # noqa: E731
    small = dict(ws=ctypes.c_void_p(16), nbytes=ctypes.c_size_t(16))
    for name, args in (("dlm_lmhead_loss", {**loss_args(V=2), "w": far(20 * MB), **small}),
                       ("dlm_lmhead_loss_grad", {**loss_grad_args(V=2), "w": far(20 * MB), **small}),
                       ("dlm_lmhead_loss_grad", {**loss_grad_args(V=2), "dw": far(20 * MB), **small})):
        assert call(name, *args.values()) == (-6 if status is None else status)


def test_clip_takes_extents_past_32_bits():
    """A flat buffer of 2^31 elements and more is taken (up to the check of overlaps, which
    ends the call here); 2^40 elements are the most, in one extent or in several."""
    big, out = T(BF16, [2 ** 31 + 5], MB), T(BF16, [2 ** 31 + 5], 3 * MB)
    assert clip([big], [out]) == -6
    assert clip([T(BF16, [2 ** 40], MB)], [T(BF16, [2 ** 40], 3 * MB)]) == -6
    assert clip([T(BF16, [2 ** 40 + 1], MB)], None) == -3
    assert clip([T(BF16, [2 ** 33, 2 ** 8], MB)], None) == -3
    assert clip([T(BF16, [2 ** 40, 2 ** 40, 2 ** 40, 2 ** 8], MB)], None) == -3    # 2^128
    assert clip([T(F32, [2 ** 31 + 5], MB)], [T(F32, [2 ** 31 + 4], 3 * MB)]) == -3


def test_empty_tensors_of_several_dimensions():
    """An empty tensor's strides say nothing (torch's of [5, 0] are 1, 1): taken as contiguous."""
    empty = [T(BF16, [5, 0], 0, [1, 1]), T(F32, [0, 4, 3], 0, [12, 3, 1]), T(F32, [2, 0, 3], 0, [3, 3, 1])]
    twice = [T(BF16, [100], 20 * MB)] * 2
    assert clip(empty + twice, empty + twice) == -6    # (the overlap of the others)
    none = dict(t=T(I32, [3, 0], 0, [1, 1]), lse=T(F32, [3, 0], 0, [1, 1]))
    rows = T(BF16, [3, 0, 64], 0, [64, 64, 1])
    assert call("dlm_lmhead_loss", *{**loss_args(), **none, "h": rows, "loss": T(F32, [0], 0)}.values()) == 0
    assert call("dlm_lmhead_loss_grad", *{**loss_grad_args(), **none, "h": rows, "dloss": T(F32, [0], 0), "dh": rows,
                                          "dw": None}.values()) == 0


def test_an_empty_tensor_may_have_any_other_extents():
    m = 2 ** 31 - 1
    big = T(BF16, [100], 20 * MB)
    for shape in ([0, m, m, m], [m, m, m, 0], [m, 0, m, m]):
        empty = T(F32, shape, 0, [0, 0, 0, 1])
        assert clip([empty, big, big], [empty, big, big]) == -6    # (the overlap of the others)
    assert clip([T(F32, [m, m, m, 1], MB)], None) == -3
