"""Where a bounded wait of the small feed-forward products runs out (DLM_CHECK_BOUNDS build), for each
kernel by itself: dx and dW alone run in launches of their own, both together in one, dW with its K
split over a cluster and without. The call ends, writes nothing outside its outputs and workspace,
and the call right behind it on the stream equals the default build's, bit for bit.

A load takes longer than 300 ns wherever its data is, so with the budgets of 100 and 300 ns every call
has waits that run out; with the longer ones the pipeline may get further before one does."""
import ctypes
import time

import pytest
import torch

from block_forms import Plans
from block_util import BF, Guarded, dev, rand
from test_gpu_block_timeout import checked  # noqa: F401

pytestmark = pytest.mark.gpu

# call, rows, width, inner width, forms: of the product, or of both gradients
CASES = [("gated", 2, 520, 2472, "few16/1"), ("gated", 17, 4328, 584, "few32/8"), ("linear", 2, 4104, 72, "few16/8"),
         ("dx1", 201, 4904, 72, "few32/1"), ("dw1", 2, 72, 392, "few128/1"), ("dw2", 9850, 136, 72, "few64/8"),
         ("dw1", 2795, 72, 2456, "few128/4"), ("both2", 390, 72, 600, "few16/4 few64/4"), ("gated", 40, 16384, 4096, "few64/4"), ("gated", 300, 8200, 1032, "few128/4"), ("gated", 66, 72, 10248, "few128/1"),
         ("linear", 40, 16384, 4096, "few64/8"), ("linear", 40, 8200, 2056, "few64/8"), ("linear", 9964, 520, 136, "few128/1"),
         ("dx1", 580, 3528, 72, "few64/1"), ("dx1", 2795, 2456, 72, "few128/1"), ("dx2", 40, 2056, 8200, "few64/8"),
         ("dw1", 515, 4264, 72, "few128/1"), ("dw2", 783, 264, 792, "few128/1"), ("dw1", 16409, 520, 328, "few64/8"),
         ("both1", 773, 264, 1672, "few128/4 few128/1"), ("both1", 857, 648, 776, "few128/2 few128/2"),
         ("both1", 740, 72, 2584, "few32/4 few128/4"), ("both2", 40, 2056, 8200, "few64/8 few128/1"),
         ("both2", 837, 1224, 200, "few128/2 few128/2")]
BUDGETS = (100, 300, 1000, 3000)


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    return Plans(str(tmp_path_factory.mktemp("plans")))


def arguments(call, N, d, f):
    """The outputs' shapes, the workspace's size, and the call on a library."""
    from paper_2608_02625_gb300 import binding as B
    x, w = rand(N, d, seed=1), [rand(f, d, seed=2 + i, std=d ** -0.5) for i in range(2)]
    dout, gate, up = (rand(N, f, seed=4 + i) for i in range(3))
    r = lambda *ts: [None if t is None else B._ref(B.describe(t)) for t in ts]  # noqa: E731
    i32 = ctypes.c_int32
    if call == "gated":
        return [(N, f)] * 3, 0, lambda lib, o, ws: lib.dlm_gated_linear(*r(x, *w), i32(1), *r(*o))
    if call == "linear":
        return [(N, f)] * 2, 0, lambda lib, o, ws: lib.dlm_linear(*r(x, w[0]), None, i32(2), *r(dout, *o), None, ctypes.c_size_t(0))
    count = int(call[-1])
    need = (B.dlm_gated_linear_grad_workspace_bytes if count == 2 else B.dlm_linear_grad_workspace_bytes)(N, f, d)
    dx, dw = call[:2] in ("dx", "bo"), call[:2] in ("dw", "bo")
    shapes = [(N, d)] * dx + [(f, d)] * (count * dw)

    def run(lib, o, ws):
        o = list(o)
        first = o.pop(0) if dx else None
        rest = o if dw else [None] * count
        tail = (ctypes.c_void_p(ws.data_ptr()), ctypes.c_size_t(need))
        if count == 2:
            return lib.dlm_gated_linear_grad(*r(dout, x, *w, gate, up), i32(1), None, *r(first, *rest), *tail)
        return lib.dlm_linear_grad(*r(dout, x, w[0], gate), i32(2), None, *r(first, *rest, None), *tail)

    return shapes, need, run


def forms(plans, call, N, d, f):
    if call == "gated":
        return plans.gated(N, d, f)
    if call == "linear":
        return plans.cols(N, d, f)
    _, x, w = plans.gradients(int(call[-1]), N, d, f)
    return {"dx": x, "dw": w, "bo": f"{x} {w}"}[call[:2]]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_a_wait_runs_out_and_nothing_is_left_behind(checked, plans, case):  # noqa: F811
    from paper_2608_02625_gb300 import binding as B
    *call, form = case
    assert forms(plans, *call) == form
    if call[0].startswith("both"):
        assert plans.gradients(int(call[0][-1]), *call[1:])[0] == "together"
    shapes, need, run = arguments(*call)
    gd = Guarded()
    ws = gd.empty(max(16, need), dtype=torch.uint8)
    want, given_up, right = ([gd.empty(*s, dtype=BF) for s in shapes] for _ in range(3))

    def bits():
        b = ctypes.c_int32(0)
        assert checked.dlm_get_device_error(ctypes.byref(b), 1) == 0
        return b.value

    B._prepare(want[0])
    assert run(B.lib, want, ws) == 0
    assert checked.dlm_set_stream(ctypes.c_void_p(torch.cuda.current_stream(dev()).cuda_stream)) == 0
    assert run(checked, right, ws) == 0  # loads the library's kernels
    torch.cuda.synchronize()
    assert bits() == 0
    ran_out = {}
    for budget in BUDGETS:
        for _ in range(4):
            t0 = time.perf_counter()
            try:
                assert checked.dlm_checked_set_wait_budget(budget) == 0
                assert run(checked, given_up, ws) == 0
            finally:
                assert checked.dlm_checked_set_wait_budget(2000000000) == 0
            assert run(checked, right, ws) == 0  # behind it, without a wait between them
            torch.cuda.synchronize()
            assert time.perf_counter() - t0 < 5.0
            got = bits()
            assert got & ~0x2 == 0
            ran_out[budget] = ran_out.get(budget, True) and bool(got & 0x2)
            for a, b in zip(right, want):
                assert torch.equal(a, b)
    gd.check()
    assert ran_out[100] and ran_out[300], ran_out
