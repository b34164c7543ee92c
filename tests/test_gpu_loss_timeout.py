"""The bounded waits of the projection loss kernels (DLM_CHECK_BOUNDS build, as in
test_checked_build.py): with a budget of 300 ns the waits on loads and MMAs run out,
the calls return with DLM_DEVERR_TIMEOUT recorded and everything torn down; with the
budget back the same calls equal the default build's, bit for bit."""
import ctypes
import time

import pytest
import torch

from train_util import dev

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.mark.parametrize("N,V,d", [(256, 4096, 2048), (1024, 4096, 2048), (2048, 5200, 2048)],
                         ids=["single_ctas", "more_rows", "pairs"])
def test_loss_pipelines_time_out_and_recover(tmp_path, N, V, d):
    from paper_2608_02625_gb300 import binding as Bn
    from paper_2608_02625_gb300 import build
    build.build(check_bounds=True, out_dir=str(tmp_path))
    lib = ctypes.CDLL(str(tmp_path / "libdlmrefine.so"))
    lib.dlm_checked_set_wait_budget.argtypes = [ctypes.c_int64]
    assert lib.dlm_set_stream(ctypes.c_void_p(torch.cuda.current_stream(dev()).cuda_stream)) == 0
    g = torch.Generator().manual_seed(N)
    h = torch.randn(N, d, generator=g).to(BF).to(dev())
    w = (torch.randn(V, d, generator=g) * d ** -0.5).to(BF).to(dev())
    t = torch.randint(-V // 4, V, (N,), generator=g, dtype=torch.int32).to(dev())
    dl = torch.full((N,), 1.0 / N, device=dev())
    ws = [torch.empty(n, dtype=torch.uint8, device=dev()) for n in (Bn.dlm_lmhead_loss_workspace_bytes(N, d),
                                                                  Bn.dlm_lmhead_loss_grad_workspace_bytes(N, V, d, 1024))]
    new = lambda: [torch.empty(N, device=dev()), torch.empty(N, device=dev()), torch.empty_like(h), torch.empty_like(w)]  # noqa: E731

    def bits():
        b = ctypes.c_int32(0)
        assert lib.dlm_get_device_error(ctypes.byref(b), 1) == 0
        return b.value

    def run(name, o, lse):
        refs = lambda *ts: [ctypes.byref(Bn.describe(x)) for x in ts]  # noqa: E731
        k = 0 if name == "loss" else 1
        args = refs(h, w, t, o[0], o[1]) if name == "loss" else refs(h, w, t, lse, dl, o[2], o[3])
        fn = lib.dlm_lmhead_loss if name == "loss" else lib.dlm_lmhead_loss_grad
        return fn(*args, ctypes.c_void_p(ws[k].data_ptr()), ctypes.c_size_t(ws[k].numel()))

    want = new()
    Bn.dlm_lmhead_loss(h, w, t, want[0], want[1], ws[0])
    Bn.dlm_lmhead_loss_grad(h, w, t, want[1], dl, want[2], want[3], ws[1])
    torch.cuda.synchronize()
    assert bits() == 0
    got = new()
    assert lib.dlm_checked_set_wait_budget(300) == 0
    try:
        for name in ("loss", "grad"):
            t0 = time.perf_counter()
            assert run(name, got, want[1]) == 0
            torch.cuda.synchronize()
            assert time.perf_counter() - t0 < 5.0, name
            assert bits() & 0x2, f"{name}: no DLM_DEVERR_TIMEOUT with a 300 ns budget"
    finally:
        assert lib.dlm_checked_set_wait_budget(2000000000) == 0
    got = new()
    assert run("loss", got, None) == 0 and run("grad", got, got[1]) == 0
    torch.cuda.synchronize()
    assert bits() == 0
    for a, b in zip(got, want):
        assert torch.equal(a, b)
