"""Host-side validation of the feed-forward block's entry points: what is refused, with
nothing launched (fake device pointers, never read)."""
import ctypes

import pytest

from test_abi import BF16, F32, I32, MB, T, U8, built  # noqa: F401
from test_abi_train import call

P, Z = ctypes.c_void_p, ctypes.c_size_t


def b(shape, at, strides=None, dt=BF16):
    return T(dt, shape, at * MB, strides)


def gated():
    return dict(x=b([6, 64], 1), wg=b([40, 64], 2), wu=b([40, 64], 3), act=1, out=b([6, 40], 4), gate=b([6, 40], 5),
                up=b([6, 40], 6))


GATED = {
    "null_x": (dict(x=None), -1), "null_wu": (dict(wu=None), -1), "null_out": (dict(out=None), -1), "gate_alone": (dict(up=None), -1),
    "x_f32": (dict(x=b([6, 64], 1, dt=F32)), -2), "out_f32": (dict(out=b([6, 40], 4, dt=F32)), -2),
    "wg_width": (dict(wg=b([40, 56], 2)), -3), "wu_rows": (dict(wu=b([48, 64], 3)), -3), "out_width": (dict(out=b([6, 48], 4)), -3),
    "out_rows": (dict(out=b([5, 40], 4)), -3), "out_rank": (dict(out=b([2, 3, 40], 4)), -3), "gate_width": (dict(gate=b([6, 64], 5)), -3),
    "d_not_of_8": (dict(x=b([6, 60], 1), wg=b([40, 60], 2), wu=b([40, 60], 3)), -3),
    "f_not_of_8": (dict(wg=b([36, 64], 2), wu=b([36, 64], 3), out=b([6, 36], 4)), -3), "rank_1": (dict(x=b([64], 1)), -3),
    "too_many": (dict(x=b([2 ** 28 + 8, 64], 1)), -3),
    "too_large": (dict(x=b([2 ** 28, 2 ** 13], 1)), -3),
    "x_apart": (dict(x=b([6, 64], 1, [128, 2])), -4), "x_overlaps_itself": (dict(x=b([6, 64], 1, [32, 1])), -4),
    "w_overlaps_itself": (dict(wg=b([40, 64], 2, [0, 1])), -4),
    "uneven_rows": (dict(x=b([2, 3, 64], 1, [1000, 64, 1])), -4), "far_rows": (dict(x=b([6, 64], 1, [2 ** 39, 1])), -4),
    "x_misaligned": (dict(x=T(BF16, [6, 64], MB + 8)), -5), "x_stride": (dict(x=b([6, 64], 1, [68, 1])), -5),
    "wg_stride": (dict(wg=b([40, 64], 2, [68, 1])), -5), "out_stride": (dict(out=b([6, 40], 4, [44, 1])), -5),
    "up_misaligned": (dict(up=T(BF16, [6, 40], 6 * MB + 2)), -5),
    "act_unknown": (dict(act=3), -6), "act_negative": (dict(act=-1), -6), "out_on_x": (dict(out=b([6, 40], 1)), -6),
    "gate_on_out": (dict(gate=T(BF16, [6, 40], 4 * MB + 16)), -6), "up_on_wu": (dict(up=b([6, 40], 3)), -6),
    "up_between_rows_too_wide": (dict(gate=b([6, 40], 5, [72, 1]), up=T(BF16, [6, 40], 5 * MB + 80, [72, 1])), -6),
    "up_on_gates_ends": (dict(gate=b([6, 40], 5, [80, 1]), up=T(BF16, [6, 40], 5 * MB + 64, [80, 1])), -6),
    "up_before_gate": (dict(gate=T(BF16, [6, 40], 5 * MB + 64, [80, 1]), up=b([6, 40], 5, [80, 1])), -6),
    "other_pitch": (dict(gate=b([6, 40], 5, [96, 1]), up=T(BF16, [6, 40], 5 * MB + 80, [88, 1])), -6),
}


@pytest.mark.parametrize("case", GATED)
def test_gated_refuses(case):
    over, status = GATED[case]
    assert call("dlm_gated_linear", *{**gated(), **over}.values()) == status


def gated_grad():
    return dict(dout=b([6, 40], 1), x=b([6, 64], 2), wg=b([40, 64], 3), wu=b([40, 64], 4), gate=b([6, 40], 5), up=b([6, 40], 6),
                act=1, add=b([6, 64], 7), dx=b([6, 64], 8), dwg=b([40, 64], 9), dwu=b([40, 64], 10), ws=P(11 * MB), n=Z(1 << 20))


GATED_GRAD = {
    "null_dout": (dict(dout=None), -1), "null_gate": (dict(gate=None), -1), "dwg_alone": (dict(dwu=None), -1),
    "nothing": (dict(add=None, dx=None, dwg=None, dwu=None), -1), "add_without_dx": (dict(dx=None), -1), "null_workspace": (dict(ws=None), -1),
    "dx_f32": (dict(dx=b([6, 64], 8, dt=F32)), -2), "add_f32": (dict(add=b([6, 64], 7, dt=F32)), -2),
    "dout_width": (dict(dout=b([6, 48], 1)), -3), "up_rows": (dict(up=b([7, 40], 6)), -3), "dx_width": (dict(dx=b([6, 56], 8)), -3),
    "add_rows": (dict(add=b([5, 64], 7)), -3), "dwu_rows": (dict(dwu=b([48, 64], 10)), -3), "dwg_width": (dict(dwg=b([40, 56], 9)), -3),
    "dout_broadcast": (dict(dout=b([6, 40], 1, [0, 1])), -4), "dout_stride": (dict(dout=b([6, 40], 1, [44, 1])), -5),
    "gate_misaligned": (dict(gate=T(BF16, [6, 40], 5 * MB + 2)), -5), "dwg_stride": (dict(dwg=b([40, 64], 9, [68, 1])), -5),
    "workspace_misaligned": (dict(ws=P(11 * MB + 8)), -5), "workspace_small": (dict(n=Z(1000)), -6), "act": (dict(act=7), -6),
    "dx_on_x": (dict(dx=b([6, 64], 2)), -6), "dx_on_part_of_add": (dict(dx=T(BF16, [6, 64], 7 * MB + 128)), -6),
    "dwg_on_wg": (dict(dwg=b([40, 64], 3)), -6), "dwu_on_dwg": (dict(dwu=b([40, 64], 9)), -6), "workspace_on_dx": (dict(ws=P(8 * MB)), -6),
    "dwu_on_add": (dict(dwu=b([40, 64], 7)), -6),
}


@pytest.mark.parametrize("case", GATED_GRAD)
def test_gated_grad_refuses(case):
    over, status = GATED_GRAD[case]
    assert call("dlm_gated_linear_grad", *{**gated_grad(), **over}.values()) == status


def linear():
    return dict(x=b([6, 64], 1), w=b([40, 64], 2), bias=T(F32, [40], 3 * MB), act=2, residual=b([6, 40], 4), out=b([6, 40], 5),
                pre=b([6, 40], 6), ws=P(7 * MB), n=Z(1 << 24))


LINEAR = {
    "null_x": (dict(x=None), -1), "null_w": (dict(w=None), -1), "null_out": (dict(out=None), -1), "bias_int": (dict(bias=T(I32, [40], 3 * MB)), -2),
    "w_f32": (dict(w=b([40, 64], 2, dt=F32)), -2), "residual_f32": (dict(residual=b([6, 40], 4, dt=F32)), -2), "pre_f32": (dict(pre=b([6, 40], 6, dt=F32)), -2),
    "bias_length": (dict(bias=T(F32, [41], 3 * MB)), -3), "w_width": (dict(w=b([40, 72], 2)), -3), "m_not_of_8": (dict(w=b([41, 64], 2)), -3),
    "out_width": (dict(out=b([6, 48], 5)), -3), "residual_rows": (dict(residual=b([1, 40], 4)), -3), "pre_rank": (dict(pre=b([2, 3, 40], 6)), -3),
    "bias_apart": (dict(bias=T(F32, [40], 3 * MB, [2])), -4), "out_overlaps_itself": (dict(out=b([6, 40], 5, [8, 1])), -4),
    "x_stride": (dict(x=b([6, 64], 1, [68, 1])), -5), "act": (dict(act=-2), -6), "out_on_x": (dict(out=b([6, 40], 1)), -6),
    "out_on_part_of_residual": (dict(out=T(BF16, [6, 40], 4 * MB + 80)), -6), "pre_on_residual": (dict(pre=b([6, 40], 4)), -6),
    "pre_on_out": (dict(pre=b([6, 40], 5)), -6), "out_on_bias": (dict(out=b([6, 40], 3)), -6),
    "residual_of_another_stride": (dict(residual=b([6, 40], 4, [48, 1]), out=b([6, 40], 4)), -6),
}


@pytest.mark.parametrize("case", LINEAR)
def test_linear_refuses(case):
    over, status = LINEAR[case]
    assert call("dlm_linear", *{**linear(), **over}.values()) == status


def linear_grad():
    return dict(dout=b([6, 40], 1), x=b([6, 64], 2), w=b([40, 64], 3), pre=b([6, 40], 4), act=2, add=b([6, 64], 5), dx=b([6, 64], 6),
                dw=b([40, 64], 7), db=T(F32, [40], 8 * MB), ws=P(9 * MB), n=Z(1 << 20))


LINEAR_GRAD = {
    "null_dout": (dict(dout=None), -1), "null_w": (dict(w=None), -1), "no_pre": (dict(pre=None), -1),
    "nothing": (dict(add=None, dx=None, dw=None, db=None), -1), "add_without_dx": (dict(dx=None), -1), "null_workspace": (dict(ws=None), -1),
    "db_int": (dict(db=T(I32, [40], 8 * MB)), -2), "dw_f32": (dict(dw=b([40, 64], 7, dt=F32)), -2), "db_length": (dict(db=T(F32, [39], 8 * MB)), -3),
    "dx_rows": (dict(dx=b([7, 64], 6)), -3), "dw_rows": (dict(dw=b([48, 64], 7)), -3), "pre_width": (dict(pre=b([6, 48], 4)), -3),
    "pre_stride": (dict(pre=b([6, 40], 4, [44, 1])), -5), "dout_misaligned": (dict(dout=T(BF16, [6, 40], MB + 2)), -5),
    "pre_without_activation": (dict(act=0), -6), "workspace_small": (dict(n=Z(100)), -6), "workspace_misaligned": (dict(ws=P(9 * MB + 8)), -5),
    "dx_on_dout": (dict(dx=b([6, 64], 1)), -6), "db_on_dw": (dict(db=T(F32, [40], 7 * MB)), -6), "dw_on_w": (dict(dw=b([40, 64], 3)), -6),
    "dx_on_part_of_add": (dict(dx=T(BF16, [6, 64], 5 * MB + 256)), -6), "workspace_on_pre": (dict(ws=P(4 * MB)), -6),
}


@pytest.mark.parametrize("case", LINEAR_GRAD)
def test_linear_grad_refuses(case):
    over, status = LINEAR_GRAD[case]
    assert call("dlm_linear_grad", *{**linear_grad(), **over}.values()) == status


def test_no_rows():
    none = lambda w, at: T(BF16, [0, w], at * MB)  # noqa: E731
    assert call("dlm_gated_linear", none(64, 1), b([40, 64], 2), b([40, 64], 3), 1, none(40, 4), None, None) == 0
    assert call("dlm_linear", none(64, 1), b([40, 64], 2), None, 0, None, none(40, 4), None, None, Z(0)) == 0


def test_workspace_sizes():
    from paper_2608_02625_gb300 import binding as B
    for size in (B.dlm_gated_linear_grad_workspace_bytes, B.dlm_linear_grad_workspace_bytes):
        assert size(0, 40, 64) == size(6, 0, 64) == size(6, 40, 60) == size(2 ** 29, 40, 64) == size(-1, 40, 64) == 0
        assert size(6, 40, 64) > 0
        assert size(2 ** 28, 2 ** 12, 8) > 2 ** 40 and size(2 ** 28, 2 ** 20, 2 ** 20) == 0
    assert B.dlm_linear_workspace_bytes(0, 40, 64) == B.dlm_linear_workspace_bytes(6, 41, 64) == 0
