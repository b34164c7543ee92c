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
    assert B.dlm_clip_grad_norm_workspace_bytes() > 0
