"""Training calls that follow each other on a stream (each kernel may be launched while
the one before it still runs) and that run at once on two streams: the same bits as with
a wait behind every call."""
import pytest
import torch

from train_util import dev

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


class Step:
    """Buffers of the last layer's training step: norm, loss, gradients, clipping, update."""

    def __init__(self, N, V, d, piece, seed):
        from paper_2608_02625_gb300 import binding as B
        g = torch.Generator(device="cpu").manual_seed(seed)
        r = lambda *s, std=1.0: (torch.randn(*s, generator=g) * std).to(dev())  # noqa: E731
        self.B, self.N, self.d = B, N, d
        self.x, self.w = r(N, d).to(BF), r(V, d, std=d ** -0.5).to(BF)
        self.nw, self.nb = 1 + r(d, std=0.2), r(d, std=0.2)
        self.t = torch.randint(-V, V, (N,), generator=g, dtype=torch.int32).to(dev())
        self.dl = torch.full((N,), 1.0 / N, device=dev())
        e = lambda *s, dtype=F32: torch.empty(*s, dtype=dtype, device=dev())  # noqa: E731
        self.h, self.mean, self.rstd, self.loss, self.lse = e(N, d, dtype=BF), e(N), e(N), e(N), e(N)
        self.dh, self.dw, self.dx, self.dnw, self.dnb = e(N, d, dtype=BF), e(V, d, dtype=BF), e(N, d, dtype=BF), e(d), e(d)
        self.norm = e(1)
        ws = lambda n: torch.empty(n, dtype=torch.uint8, device=dev())  # noqa: E731
        self.ws = [ws(B.dlm_lmhead_loss_workspace_bytes(N, d)), ws(B.dlm_lmhead_loss_grad_workspace_bytes(N, V, d, piece)),
                   ws(B.dlm_layer_norm_grad_workspace_bytes(N, d)), ws(B.dlm_clip_grad_norm_workspace_bytes())]

    def calls(self):
        B, grads = self.B, [self.dw, self.dnw, self.dnb]
        yield lambda: B.dlm_layer_norm(self.x, self.nw, self.nb, 1e-5, self.h, self.mean, self.rstd)
        yield lambda: B.dlm_lmhead_loss(self.h, self.w, self.t, self.loss, self.lse, self.ws[0])
        yield lambda: B.dlm_lmhead_loss_grad(self.h, self.w, self.t, self.lse, self.dl, self.dh, self.dw, self.ws[1])
        yield lambda: B.dlm_layer_norm_grad(self.dh, self.x, self.nw, self.mean, self.rstd, self.dx, self.dnw, self.dnb, self.ws[2])
        yield lambda: B.dlm_clip_grad_norm(grads, grads, 0.05, self.norm, self.ws[3])

    def update(self):
        for p, g in ((self.w, self.dw), (self.nw, self.dnw), (self.nb, self.dnb), (self.x, self.dx)):
            p.sub_(g, alpha=0.5)

    def seen(self):
        return [t.clone() for t in (self.loss, self.lse, self.dh, self.dw, self.dx, self.dnw, self.dnb, self.norm, self.w)]


SIZES = [(1, 40, 8, 256), (130, 2001, 64, 1024), (600, 3000, 512, 1024), (1030, 1500, 1024, 0)]


def run(size, sync, seed=1):
    s, seen = Step(*size, seed), []
    for _ in range(3):
        for call in s.calls():
            call()
            if sync:
                torch.cuda.synchronize()
        seen += s.seen()
        s.update()
    torch.cuda.synchronize()
    assert s.B.device_error(clear=True) == 0
    return seen


@pytest.mark.parametrize("size", SIZES, ids=str)
def test_results_do_not_depend_on_waiting_between_calls(size):
    waited = run(size, True)
    for _ in range(3):
        for a, b in zip(run(size, False), waited):
            assert torch.equal(a, b)


@pytest.mark.parametrize("size", SIZES[1:], ids=str)
def test_two_streams_at_once(size):
    want = [run(size, True, seed) for seed in (1, 2)]
    steps = [Step(*size, seed) for seed in (1, 2)]
    streams = [torch.cuda.Stream(dev()) for _ in steps]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(3):
        for k, calls in enumerate(zip(*(s.calls() for s in steps))):
            for call, stream in zip(calls, streams):
                with torch.cuda.stream(stream):
                    call()
        for s, stream, out in zip(steps, streams, got):
            with torch.cuda.stream(stream):
                out += s.seen()
                s.update()
    torch.cuda.synchronize()
    assert steps[0].B.device_error(clear=True) == 0
    for g, w in zip(got, want):
        for a, b in zip(g, w):
            assert torch.equal(a, b)


def test_two_graphs_with_one_workspace():
    """Two recorded calls of other sizes that share a workspace, replayed in turn."""
    steps = [Step(600, 3000, 512, 1024, 5), Step(130, 2001, 512, 1024, 6)]
    want = []
    for s in steps:
        for call in s.calls():
            call()
        want.append(s.seen())
    steps[1].ws = steps[0].ws
    graphs = []
    torch.cuda.synchronize()
    for s in steps:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            for call in s.calls():
                call()
        graphs.append(g)
    for _ in range(3):
        for g in graphs:
            g.replay()
    torch.cuda.synchronize()
    assert steps[0].B.device_error(clear=True) == 0
    for s, w in zip(steps, want):
        got = s.seen()
        # the workspace of the larger call allows the smaller one other pieces
        for k, (a, b) in enumerate(zip(got, w)):
            if s is steps[0] or k < 2:
                assert torch.equal(a, b)
            else:
                assert float((a.double() - b.double()).norm()) <= 2.0 ** -7 * float(b.double().norm())
