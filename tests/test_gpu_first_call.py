"""The first call of a host thread, which has no context of its own yet, is the library's."""
import threading

import pytest
import torch

from train_util import dev

pytestmark = pytest.mark.gpu


def rand(*shape):
    return torch.randn(*shape, device=dev()).to(torch.bfloat16)


def empty(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype, device=dev())


def attention(B):
    q, k, v, n = rand(1, 64, 4, 128), rand(1, 64, 2, 128), rand(1, 64, 2, 128), torch.tensor([64], dtype=torch.int32, device=dev())
    out = empty(1, 64, 4, 128)
    return lambda: (B.dlm_bidir_attn(q, k, v, n, out),), (out,)


def confidence(B):
    h, w = rand(20, 128), rand(300, 128)
    outs = empty(20, dtype=torch.int32), empty(20, dtype=torch.float32), empty(20, dtype=torch.float32)
    ws = empty(B.dlm_lmhead_workspace_bytes(20), dtype=torch.uint8)
    return lambda: B.dlm_lmhead_confidence(h, w, *outs, ws), outs


def loss(B):
    h, w, t = rand(20, 128), rand(300, 128), torch.arange(20, dtype=torch.int32, device=dev())
    outs = empty(20, dtype=torch.float32), empty(20, dtype=torch.float32)
    ws = empty(B.dlm_lmhead_loss_workspace_bytes(20, 128), dtype=torch.uint8)
    return lambda: B.dlm_lmhead_loss(h, w, t, *outs, ws), outs


def gated(B):
    x, wg, wu = rand(20, 128), rand(72, 128), rand(72, 128)
    outs = empty(20, 72), empty(20, 72), empty(20, 72)
    return lambda: B.dlm_gated_linear(x, wg, wu, B.ACT_SILU, *outs), outs


def gated_gradients(B):
    x, wg, wu, dout, gate, up = rand(20, 128), rand(72, 128), rand(72, 128), rand(20, 72), rand(20, 72), rand(20, 72)
    outs = empty(20, 128), empty(72, 128), empty(72, 128)
    ws = empty(B.dlm_gated_linear_grad_workspace_bytes(20, 72, 128), dtype=torch.uint8)
    return lambda: B.dlm_gated_linear_grad(dout, x, wg, wu, gate, up, B.ACT_SILU, None, *outs, ws), outs


def linear(B):
    x, w = rand(20, 128), rand(72, 128)
    out = empty(20, 72)
    return lambda: B.dlm_linear(x, w, None, B.ACT_NONE, None, out, None, None), (out,)


def linear_gradients(B):
    x, w, dout = rand(20, 128), rand(72, 128), rand(20, 72)
    outs = empty(20, 128), empty(72, 128)
    ws = empty(B.dlm_linear_grad_workspace_bytes(20, 72, 128), dtype=torch.uint8)
    return lambda: B.dlm_linear_grad(dout, x, w, None, B.ACT_NONE, None, *outs, None, ws), outs


@pytest.mark.parametrize("make", [attention, confidence, loss, gated, gated_gradients, linear, linear_gradients], ids=lambda f: f.__name__)
def test_first_call_of_a_thread(make):
    from paper_2608_02625_gb300 import binding as B
    torch.manual_seed(1)
    call, outs = make(B)
    call()
    want = [t.clone() for t in outs]
    for t in outs:
        t.zero_()
    torch.cuda.synchronize()
    wrong = []

    def work():
        try:
            call()
        except Exception as e:  # noqa: BLE001
            wrong.append(e)

    thread = threading.Thread(target=work)
    thread.start()
    thread.join()
    torch.cuda.synchronize()
    assert not wrong and B.device_error(clear=True) == 0
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
