"""Where a bounded wait of the feed-forward products runs out (DLM_CHECK_BOUNDS build), early or
late in the launch, in any of its roles: the call ends, writes nothing outside its outputs and
workspace, and leaves nothing on its way: the call right behind it on the stream equals the default
build's, bit for bit. Sizes for each kernel: pairs of CTAs for thousands of rows, single CTAs in
clusters for a few, both gradients in one launch where they are small, and apart."""
import ctypes
import time

import pytest
import torch

from block_util import BF, F32, Guarded, dev, rand

pytestmark = pytest.mark.gpu

# rows, width, inner width
SIZES = {"pairs": (3000, 1024, 2048), "few": (20, 2048, 1032), "few_apart": (40, 2048, 8192), "long": (700, 64, 2048)}
CALLS = ("gated", "gated_grad", "linear", "linear_grad")


@pytest.fixture(scope="module")
def checked(tmp_path_factory):
    from paper_2608_02625_gb300 import build
    out = tmp_path_factory.mktemp("checked")
    build.build(check_bounds=True, out_dir=str(out))
    lib = ctypes.CDLL(str(out / "libdlmrefine.so"))
    lib.dlm_checked_set_wait_budget.argtypes = [ctypes.c_int64]
    return lib


def arguments(name, size):
    """Inputs of a call, the shapes of its outputs, its workspace's size, and the call on a library."""
    from paper_2608_02625_gb300 import binding as B
    N, d, f = SIZES[size]
    x, wg, wu = rand(N, d, seed=1), rand(f, d, seed=2, std=d ** -0.5), rand(f, d, seed=3, std=d ** -0.5)
    dout, gate, up = rand(N, f, seed=4), rand(N, f, seed=5), rand(N, f, seed=6)
    shapes = {"gated": [(N, f)] * 3, "gated_grad": [(N, d), (f, d), (f, d)], "linear": [(N, f), (N, f)], "linear_grad": [(N, d), (f, d), (f,)]}[name]
    need = {"gated": 0, "gated_grad": B.dlm_gated_linear_grad_workspace_bytes(N, f, d), "linear": B.dlm_linear_workspace_bytes(N, f, d),
            "linear_grad": B.dlm_linear_grad_workspace_bytes(N, f, d)}[name]

    def run(lib, o, ws):
        r = lambda *ts: [B._ref(B.describe(t)) for t in ts]  # noqa: E731
        w = (ctypes.c_void_p(ws.data_ptr()), ctypes.c_size_t(need))
        i = ctypes.c_int32
        if name == "gated":
            return lib.dlm_gated_linear(*r(x, wg, wu), i(1), *r(*o))
        if name == "gated_grad":
            return lib.dlm_gated_linear_grad(*r(dout, x, wg, wu, gate, up), i(1), None, *r(*o), *w)
        if name == "linear":
            return lib.dlm_linear(*r(x, wg), None, i(2), *r(dout, *o), *w)
        return lib.dlm_linear_grad(*r(dout, x, wg, gate), i(2), None, *r(*o), *w)

    return shapes, need, run


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("budget", [100, 300, 1000, 3000, 10000])
def test_nothing_is_left_behind(checked, budget, size, name):
    from paper_2608_02625_gb300 import binding as B
    shapes, need, run = arguments(name, size)
    gd = Guarded()
    ws = gd.empty(max(16, need), dtype=torch.uint8)
    outs = lambda g=gd: [g.empty(*s, dtype=BF if len(s) == 2 else F32) for s in shapes]  # noqa: E731

    def bits():
        b = ctypes.c_int32(0)
        assert checked.dlm_get_device_error(ctypes.byref(b), 1) == 0
        return b.value

    want, given_up, right = outs(), outs(), outs()
    B._prepare(want[0])
    assert run(B.lib, want, ws) == 0
    assert checked.dlm_set_stream(ctypes.c_void_p(torch.cuda.current_stream(dev()).cuda_stream)) == 0
    assert run(checked, right, ws) == 0  # loads the library's kernels
    torch.cuda.synchronize()
    bits()
    for _ in range(2):
        t0 = time.perf_counter()
        try:
            assert checked.dlm_checked_set_wait_budget(budget) == 0
            assert run(checked, given_up, ws) == 0
        finally:
            assert checked.dlm_checked_set_wait_budget(2000000000) == 0
        assert run(checked, right, ws) == 0  # behind it, without a wait between them
        torch.cuda.synchronize()
        assert time.perf_counter() - t0 < 5.0
        # (The GPU's timer goes in steps of about a microsecond, as long as the waits of the smaller
        # calls, all of whose CTAs begin at once: there none or all of them run out.)
        assert bits() & 0x2 or budget > 300 or size != "pairs", f"no wait of {budget} ns ran out"
        for a, b in zip(right, want):
            assert torch.equal(a, b)
    gd.check()
