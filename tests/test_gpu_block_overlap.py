"""The feed-forward block in a training step: chains of calls without waits between them, two
streams, two threads, captured graphs that share a workspace, and the whole step against fp64 autograd."""
import threading

import pytest
import torch

from block_util import BF, F32, dev, rand

pytestmark = pytest.mark.gpu


class Step:
    """x -> gated block (+ x) -> layer norm -> loss; gradients back; the norm over all of them; AdamW."""

    def __init__(self, N, V, d, f, seed, eight=False):
        from paper_2608_02625_gb300 import binding as B
        self.B, self.N, self.V, self.d, self.f = B, N, V, d, f
        r = lambda *s, std=1.0, k=0: rand(*s, seed=seed * 100 + k, std=std)  # noqa: E731
        e = lambda *s, t=BF: torch.empty(*s, dtype=t, device=dev())  # noqa: E731
        self.x = r(N, d, k=1)
        self.weights = [r(f, d, std=d ** -0.5, k=2), r(f, d, std=d ** -0.5, k=3), r(d, f, std=f ** -0.5, k=4), r(V, d, std=d ** -0.5, k=5),
                        r(d, std=0.1, k=6) + 1, r(d, std=0.1, k=7), r(d, std=0.1, k=8)]
        self.masters = [w.float() for w in self.weights]
        self.grads = [e(*w.shape) for w in self.weights]
        g = torch.Generator().manual_seed(seed)
        self.t = torch.randint(-V // 2, V, (N,), generator=g, dtype=torch.int32).to(dev())
        self.dl = torch.full((N,), 1.0 / N, device=dev())
        self.gate, self.up, self.h, self.dh = e(N, f), e(N, f), e(N, f), e(N, f)
        self.y, self.n, self.dn, self.dy, self.dx = e(N, d), e(N, d), e(N, d), e(N, d), e(N, d)
        self.mean, self.rstd, self.loss, self.lse = (e(N, t=F32) for _ in range(4))
        self.norm, self.lr, self.step = e(1, t=F32), torch.full((1,), 1e-2, device=dev()), torch.ones(1, dtype=torch.int32, device=dev())
        st = torch.uint8 if eight else F32
        self.m, self.v = ([torch.zeros(w.shape, dtype=st, device=dev()) for w in self.weights] for _ in range(2))
        self.ms, self.vs = ([torch.zeros((w.numel() + 255) // 256, device=dev()) for w in self.weights] if eight else None for _ in range(2))
        self.hyper = B.AdamwParams(lr=self.lr, step=self.step, norm=self.norm, max_norm=0.5, weight_decay=0.1)
        need = [B.dlm_linear_workspace_bytes(N, d, f), B.dlm_lmhead_loss_workspace_bytes(N, d),
                B.dlm_lmhead_loss_grad_workspace_bytes(N, V, d), B.dlm_layer_norm_grad_workspace_bytes(N, d),
                B.dlm_linear_grad_workspace_bytes(N, d, f), B.dlm_gated_linear_grad_workspace_bytes(N, f, d),
                B.dlm_clip_grad_norm_workspace_bytes()]
        self.ws = torch.empty(max(need), dtype=torch.uint8, device=dev())  # one for every call: they follow each other

    def calls(self):
        B, ws = self.B, self.ws
        wg, wu, wd, wv, bd, nw, nb = self.weights
        gg, gu, gdn, gv, gb, gnw, gnb = self.grads
        yield lambda: B.dlm_gated_linear(self.x, wg, wu, B.ACT_SILU, self.h, self.gate, self.up)
        yield lambda: B.dlm_linear(self.h, wd, bd, B.ACT_NONE, self.x, self.y, None, ws)
        yield lambda: B.dlm_layer_norm(self.y, nw, nb, 1e-5, self.n, self.mean, self.rstd)
        yield lambda: B.dlm_lmhead_loss(self.n, wv, self.t, self.loss, self.lse, ws)
        yield lambda: B.dlm_lmhead_loss_grad(self.n, wv, self.t, self.lse, self.dl, self.dn, gv, ws)
        yield lambda: B.dlm_layer_norm_grad(self.dn, self.y, nw, self.mean, self.rstd, self.dy, gnw, gnb, ws)
        yield lambda: B.dlm_linear_grad(self.dy, self.h, wd, None, B.ACT_NONE, None, self.dh, gdn, gb, ws)
        yield lambda: B.dlm_gated_linear_grad(self.dh, self.x, wg, wu, self.gate, self.up, B.ACT_SILU, self.dy, self.dx, gg, gu, ws)
        yield lambda: B.dlm_clip_grad_norm(self.grads, None, 0.5, self.norm, ws)
        yield lambda: B.dlm_adamw(self.weights, self.masters, self.grads, self.m, self.v, self.ms, self.vs, self.hyper)
        yield lambda: self.step.add_(1)

    def state(self):
        return [self.y, self.loss, self.lse, self.dx, self.norm, *self.grads, *self.weights, *self.masters, *self.m, *self.v]

    def seen(self):
        return [t.clone() for t in self.state()]


SIZES = [(1, 40, 8, 16), (20, 300, 136, 264), (130, 2001, 64, 1000), (600, 3000, 512, 1032)]


def run(size, sync, seed=1, eight=False):
    s, seen = Step(*size, seed, eight), []
    for _ in range(3):
        for call in s.calls():
            call()
            if sync:
                torch.cuda.synchronize()
        seen += s.seen()
    torch.cuda.synchronize()
    assert s.B.device_error(clear=True) == 0
    return seen


@pytest.mark.parametrize("eight", [False, True], ids=["32bit", "8bit"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_results_do_not_depend_on_waiting_between_calls(size, eight):
    waited = run(size, True, eight=eight)
    for _ in range(3):
        for a, b in zip(run(size, False, eight=eight), waited):
            assert torch.equal(a, b)


@pytest.mark.parametrize("size", SIZES[1:], ids=str)
def test_two_streams_at_once(size):
    want = [run(size, True, seed) for seed in (1, 2)]
    steps = [Step(*size, seed) for seed in (1, 2)]
    streams = [torch.cuda.Stream(dev()) for _ in steps]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(3):
        for calls in zip(*(s.calls() for s in steps)):
            for call, stream in zip(calls, streams):
                with torch.cuda.stream(stream):
                    call()
        for s, stream, out in zip(steps, streams, got):
            with torch.cuda.stream(stream):
                out += s.seen()
    torch.cuda.synchronize()
    assert steps[0].B.device_error(clear=True) == 0
    for g, w in zip(got, want):
        for a, b in zip(g, w):
            assert torch.equal(a, b)


def test_two_threads_at_once():
    """Each thread its own stream, its own step."""
    size = SIZES[2]
    want = [run(size, True, seed) for seed in (1, 2)]
    steps = [Step(*size, seed) for seed in (1, 2)]
    torch.cuda.synchronize()
    got, wrong = [[], []], []

    def work(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream(dev())):
                for _ in range(3):
                    for call in steps[i].calls():
                        call()
                    got[i] += steps[i].seen()
        except Exception as e:  # noqa: BLE001
            wrong.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not wrong and steps[0].B.device_error(clear=True) == 0
    for g, w in zip(got, want):
        assert len(g) == len(w) and all(torch.equal(a, b) for a, b in zip(g, w))


def test_two_graphs_with_one_workspace():
    """Two recorded steps of other sizes that share a workspace, replayed in turn: three steps each."""
    sizes = [(600, 3000, 512, 1032), (40, 2001, 136, 264)]
    want = [run(size, True) for size in sizes]
    steps = [Step(*size, 1) for size in sizes]
    steps[0].ws = steps[1].ws = max((s.ws for s in steps), key=lambda t: t.numel())
    # the loss's gradients go through the vocabulary in pieces that the workspace allows; here one holds all
    graphs = []
    torch.cuda.synchronize()
    for s in steps:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            for call in s.calls():
                call()
        graphs.append(g)
    got = [[], []]
    for _ in range(3):
        for g, s, out in zip(graphs, steps, got):
            g.replay()
            out += s.seen()
    torch.cuda.synchronize()
    assert steps[0].B.device_error(clear=True) == 0
    for g, w in zip(got, want):
        for a, b in zip(g, w):
            assert torch.equal(a, b)


@pytest.mark.parametrize("size", [(20, 300, 136, 264), (300, 1000, 256, 520)], ids=str)
def test_a_step_is_fp64_autograds(size):
    """All gradients of the step against fp64 autograd through the same bf16 weights: intermediate
    results are rounded to bf16 at five places on the way, so within 4 % of their norm each
    (2^-8 for each rounding, grown by the norm's 1 / std and the sums behind it)."""
    s = Step(*size, 3)
    before = [w.double().requires_grad_() for w in s.weights]
    x = s.x.double().requires_grad_()
    for call in list(s.calls())[:9]:
        call()
    torch.cuda.synchronize()
    wg, wu, wd, wv, bd, nw, nb = before
    h = torch.nn.functional.silu(x @ wg.T) * (x @ wu.T)
    y = h @ wd.T + bd + x
    n = torch.nn.functional.layer_norm(y, (s.d,), nw, nb, 1e-5)
    rows = (s.t >= 0) & (s.t < s.V)
    loss = torch.nn.functional.cross_entropy((n @ wv.T)[rows], s.t[rows].long(), reduction="sum") / s.N
    loss.backward()
    for got, want, name in zip([s.dx, *s.grads], [x.grad, *(w.grad for w in before)], ("x", "wg", "wu", "wd", "wv", "bd", "nw", "nb")):
        off = float((got.double() - want).norm() / want.norm())
        assert off <= 0.04, (name, off)
    total = sum(float((w.grad ** 2).sum()) for w in before) ** 0.5
    assert abs(float(s.norm) - total) <= 0.02 * total
