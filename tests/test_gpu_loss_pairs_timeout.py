"""Where a bounded wait of a pair of CTAs runs out (DLM_CHECK_BOUNDS build, as in
test_gpu_loss_timeout.py), early or late in the launch, in any of its roles: the call ends,
writes nothing outside its outputs and workspace, and leaves nothing on its way: the call
right behind it on the stream equals the default build's, bit for bit."""
import ctypes
import time

import pytest
import torch

from test_gpu_loss_pairs import plan
from train_util import Guarded, dev

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
N, V, D, PIECE = 800, 11000, 2048, 4096
CALLS = ("loss", "both", "d_hidden", "d_weight")


@pytest.fixture(scope="module")
def checked(tmp_path_factory):
    from paper_2608_02625_gb300 import build
    out = tmp_path_factory.mktemp("checked")
    build.build(check_bounds=True, out_dir=str(out))
    lib = ctypes.CDLL(str(out / "libdlmrefine.so"))
    lib.dlm_checked_set_wait_budget.argtypes = [ctypes.c_int64]
    return lib


@pytest.fixture(scope="module")
def case():
    """Inputs, and the default build's results."""
    from paper_2608_02625_gb300 import binding as B
    g = torch.Generator().manual_seed(3)
    h = torch.randn(N, D, generator=g).to(BF).to(dev())
    w = (torch.randn(V, D, generator=g) * D ** -0.5).to(BF).to(dev())
    t = torch.randint(0, V, (N,), generator=g, dtype=torch.int32)
    t[::40] = -1
    t, dl = t.to(dev()), torch.full((N,), 1.0 / N, device=dev())
    ws = [torch.empty(k, dtype=torch.uint8, device=dev()) for k in (B.dlm_lmhead_loss_workspace_bytes(N, D),
                                                                  B.dlm_lmhead_loss_grad_workspace_bytes(N, V, D, PIECE))]
    loss, lse = torch.empty(N, device=dev()), torch.empty(N, device=dev())
    want = {}
    B.dlm_lmhead_loss(h, w, t, loss, lse, ws[0])
    want["loss"] = (loss, lse)
    for name in CALLS[1:]:
        dh, dw = (None if name == "d_weight" else torch.empty_like(h)), (None if name == "d_hidden" else torch.empty_like(w))
        B.dlm_lmhead_loss_grad(h, w, t, lse, dl, dh, dw, ws[1])
        want[name] = (dh, dw)
    torch.cuda.synchronize()
    assert [plan(x)[1] for x in ws] == [1, 1]
    return h, w, t, dl, lse, want


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("budget", [100, 300, 1000, 3000, 10000, 30000])
def test_nothing_is_left_behind(checked, case, budget, name):
    from paper_2608_02625_gb300 import binding as B
    h, w, t, dl, lse, want = case
    gd = Guarded()
    own = B.dlm_lmhead_loss_workspace_bytes(N, D) if name == "loss" else B.dlm_lmhead_loss_grad_workspace_bytes(N, V, D, PIECE)
    ws = gd.empty(own, dtype=torch.uint8)

    def outs():
        if name == "loss":
            return gd.empty(N), gd.empty(N)
        return (None if name == "d_weight" else gd.empty(N, D, dtype=BF)), (None if name == "d_hidden" else gd.empty(V, D, dtype=BF))

    def run(o):
        ts = (h, w, t, *o) if name == "loss" else (h, w, t, lse, dl, *o)
        fn = checked.dlm_lmhead_loss if name == "loss" else checked.dlm_lmhead_loss_grad
        refs = [B._ref(B.describe(x)) for x in ts]
        return fn(*refs, ctypes.c_void_p(ws.data_ptr()), ctypes.c_size_t(ws.numel()))

    def bits():
        b = ctypes.c_int32(0)
        assert checked.dlm_get_device_error(ctypes.byref(b), 1) == 0
        return b.value

    assert checked.dlm_set_stream(ctypes.c_void_p(torch.cuda.current_stream(dev()).cuda_stream)) == 0
    given_up, right = outs(), outs()
    assert run(right) == 0  # loads the library's kernels
    torch.cuda.synchronize()
    bits()
    for _ in range(2):
        t0 = time.perf_counter()
        try:
            assert checked.dlm_checked_set_wait_budget(budget) == 0
            assert run(given_up) == 0
        finally:
            assert checked.dlm_checked_set_wait_budget(2000000000) == 0
        assert run(right) == 0  # behind it, without a wait between them
        torch.cuda.synchronize()
        assert time.perf_counter() - t0 < 5.0
        assert bits() & 0x2 or budget > 1000, f"no wait of {budget} ns ran out"
        for a, b in zip(right, want[name]):
            assert a is None or torch.equal(a, b)
    gd.check()
