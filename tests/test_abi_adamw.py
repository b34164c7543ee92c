"""Host-side validation of dlm_adamw: what is refused, with nothing launched (fake device
pointers, never read), and the layout of its parameters."""
import ctypes
import os
import shutil
import subprocess

import pytest

from test_abi import BF16, F32, I32, MB, ROOT, T, U8, built  # noqa: F401


def hyper(**over):
    from paper_2608_02625_gb300.binding import DlmAdamwParams
    h = dict(beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.1, max_norm=1.0, lr=100 * MB, step=101 * MB, norm=102 * MB)
    h.update(over)
    return DlmAdamwParams(**h)


def lists(eight=False, masters=True):
    st = U8 if eight else F32
    a = dict(params=[T(BF16, [300], 1 * MB), T(BF16, [7, 3], 2 * MB)], masters=[T(F32, [300], 3 * MB), T(F32, [7, 3], 4 * MB)],
             grads=[T(F32, [300], 5 * MB), T(BF16, [7, 3], 6 * MB)], m=[T(st, [300], 7 * MB), T(st, [7, 3], 8 * MB)],
             v=[T(st, [300], 9 * MB), T(st, [7, 3], 10 * MB)], ms=None, vs=None)
    if eight:
        a.update(ms=[T(F32, [2], 11 * MB), T(F32, [1], 12 * MB)], vs=[T(F32, [2], 13 * MB), T(F32, [1], 14 * MB)])
    if not masters:
        a.update(masters=None)
    return a


def call(a, h=None, count=2):
    from paper_2608_02625_gb300.binding import DlmTensor, lib
    arr = [None if x is None else (DlmTensor * max(1, len(x)))(*x) for x in a.values()]
    h = hyper() if h is None else h
    return lib.dlm_adamw(*arr, count, ctypes.byref(h) if h != "null" else None)


LISTS = {
    "no_params": (dict(params=None), -1), "no_grads": (dict(grads=None), -1), "no_m": (dict(m=None), -1),
    "no_v": (dict(v=None), -1), "one_scale_list": (dict(ms=[T(F32, [2], 11 * MB), T(F32, [1], 12 * MB)]), -1),
    "params_f32_beside_masters": (dict(params=[T(F32, [300], MB), T(BF16, [7, 3], 2 * MB)]), -2),
    "masters_bf16": (dict(masters=[T(BF16, [300], 3 * MB), T(F32, [7, 3], 4 * MB)]), -2),
    "grad_int": (dict(grads=[T(I32, [300], 5 * MB), T(BF16, [7, 3], 6 * MB)]), -2),
    "m_codes_without_scales": (dict(m=[T(U8, [300], 7 * MB), T(F32, [7, 3], 8 * MB)]), -2),
    "v_bf16": (dict(v=[T(F32, [300], 9 * MB), T(BF16, [7, 3], 10 * MB)]), -2),
    "params_shape": (dict(params=[T(BF16, [300], MB), T(BF16, [3, 7], 2 * MB)]), -3),
    "v_shape": (dict(v=[T(F32, [301], 9 * MB), T(F32, [7, 3], 10 * MB)]), -3),
    "too_large": ({k: [T(t, [2 ** 31 - 1, 2 ** 10], p * MB), T(t, [7, 3], (p + 1) * MB)] for k, t, p in
                   (("params", BF16, 1), ("masters", F32, 3), ("grads", F32, 5), ("m", F32, 7), ("v", F32, 9))}, -3),
    "m_not_contiguous": (dict(m=[T(F32, [300], 7 * MB), T(F32, [7, 3], 8 * MB, [4, 1])]), -4),
    "grad_misaligned": (dict(grads=[T(F32, [300], 5 * MB + 2), T(BF16, [7, 3], 6 * MB)]), -5),
    "m_on_v": (dict(m=[T(F32, [300], 9 * MB), T(F32, [7, 3], 8 * MB)]), -6),
    "params_on_grads": (dict(params=[T(BF16, [300], 5 * MB + 100), T(BF16, [7, 3], 2 * MB)]), -6),
    "same_params_twice": (dict(params=[T(BF16, [300], MB), T(BF16, [7, 3], MB)]), -6),
    "m_on_lr": (dict(m=[T(F32, [300], 100 * MB - 8), T(F32, [7, 3], 8 * MB)]), -6),
    "masters_on_step": (dict(masters=[T(F32, [300], 101 * MB), T(F32, [7, 3], 4 * MB)]), -6),
    "v_on_norm": (dict(v=[T(F32, [300], 102 * MB - 1196), T(F32, [7, 3], 10 * MB)]), -6),
}


@pytest.mark.parametrize("case", LISTS)
def test_refuses_tensors(case):
    over, status = LISTS[case]
    assert call({**lists(), **over}) == status


EIGHT = {
    "m_f32": (dict(m=[T(F32, [300], 7 * MB), T(U8, [7, 3], 8 * MB)]), -2),
    "scales_bf16": (dict(ms=[T(BF16, [2], 11 * MB), T(F32, [1], 12 * MB)]), -2),
    "scales_short": (dict(ms=[T(F32, [1], 11 * MB), T(F32, [1], 12 * MB)]), -3),
    "scales_long": (dict(vs=[T(F32, [2], 13 * MB), T(F32, [2], 14 * MB)]), -3),
    "scales_apart": (dict(vs=[T(F32, [2], 13 * MB, [2]), T(F32, [1], 14 * MB)]), -4),
    "scales_on_codes": (dict(ms=[T(F32, [2], 7 * MB + 296), T(F32, [1], 12 * MB)]), -6),
}


@pytest.mark.parametrize("case", EIGHT)
def test_refuses_codes(case):
    over, status = EIGHT[case]
    assert call({**lists(True), **over}) == status


@pytest.mark.parametrize("over,status", [
    (dict(lr=None), -1), (dict(step=None), -1), (dict(beta1=1.0), -6), (dict(beta2=-0.1), -6), (dict(beta1=float("nan")), -6),
    (dict(eps=-1e-8), -6), (dict(eps=float("inf")), -6), (dict(weight_decay=float("nan")), -6), (dict(max_norm=-1.0), -6),
    (dict(max_norm=float("nan")), -6), (dict(lr=100 * MB + 2), -5), (dict(step=101 * MB + 1), -5), (dict(norm=102 * MB + 3), -5)])
def test_refuses_parameters(over, status):
    assert call(lists(), hyper(**over)) == status


def test_refuses_counts_and_no_parameters():
    assert call(lists(), "null") == -1
    assert call(lists(), count=-1) == -6
    assert call(lists(), count=20000) == -6


def test_nothing_to_do():
    empty = {k: [T(t, [0], 0)] for k, t in (("params", F32), ("masters", F32), ("grads", F32), ("m", F32), ("v", F32))}
    empty.update(masters=None, ms=None, vs=None)
    assert call(empty, count=1) == 0
    assert call(dict.fromkeys(lists()), count=0) == 0


def test_the_binding_refuses_lists_of_other_lengths():
    from paper_2608_02625_gb300 import binding as B
    with pytest.raises((ValueError, AttributeError)):
        B.dlm_adamw([1], None, [], [], [], None, None, B.AdamwParams(None, None))


def test_the_binding_refuses_scalars_that_are_missing_or_on_the_host():
    import torch

    from paper_2608_02625_gb300 import binding as B
    for lr, step in ((None, None), (torch.ones(1), None), (torch.ones(1), torch.ones(1, dtype=torch.int32))):
        with pytest.raises(ValueError):
            B.AdamwParams(lr, step).to_c()


SRC = r"""
#include <stddef.h>
#include <stdio.h>
#include "dlmrefine.h"
int main(void) {
  printf("%zu %zu %zu %zu %zu %zu %zu %zu %zu\n", sizeof(dlm_adamw_params), offsetof(dlm_adamw_params, beta1),
         offsetof(dlm_adamw_params, beta2), offsetof(dlm_adamw_params, eps), offsetof(dlm_adamw_params, weight_decay),
         offsetof(dlm_adamw_params, max_norm), offsetof(dlm_adamw_params, lr), offsetof(dlm_adamw_params, step),
         offsetof(dlm_adamw_params, norm));
  return DLM_ADAMW_BLOCK == 256 ? 0 : 1;
}
"""


def test_layout_matches_the_header(tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if not cc:
        pytest.skip("no C compiler")
    (tmp_path / "layout.c").write_text(SRC)
    exe = str(tmp_path / "layout")
    subprocess.run([cc, "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(tmp_path / "layout.c"), "-o", exe],
                   check=True)
    got = [int(x) for x in subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split()]
    from paper_2608_02625_gb300 import binding as B
    P = B.DlmAdamwParams
    assert got == [ctypes.sizeof(P)] + [getattr(P, n).offset for n in ("beta1", "beta2", "eps", "weight_decay", "max_norm", "lr",
                                                                     "step", "norm")]
    assert B.ADAMW_BLOCK == 256
