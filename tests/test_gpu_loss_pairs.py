"""The projection loss and its gradients where CTAs work in pairs: calls that follow each
other without a wait, two streams at once, graphs that share a workspace, and one captured
call over the numbers of scored rows between which the form changes. What ran is read from
the start of the workspace (the scored rows, and whether pairs took them), so that a later
rule for the choice cannot take the pairs out of these tests unseen."""
import pytest
import torch

from test_gpu_lmhead_loss import STEP
from test_gpu_train_overlap import Step
from train_util import U32, dev

pytestmark = pytest.mark.gpu
BF = torch.bfloat16

# Of these N rows about half are scored (targets are drawn from [-V, V)): above 384, and n V d
# above 16e9.
PAIRS = (1300, 16000, 2048, 0)
PIECES = (1400, 14000, 2048, 4096)
# Rows enough that pairs may work, and too few scored ones: both forms are launched.
FEW = (700, 20000, 2048, 0)


def plan(ws):
    """(scored rows, whether pairs took them) of the call that used the workspace last."""
    n, pairs = ws[:8].view(torch.int32).tolist()
    return n, pairs


def steps_of(step, sync=False):
    seen = []
    for _ in range(3):
        for call in step.calls():
            call()
            if sync:
                torch.cuda.synchronize()
        seen += step.seen()
        step.update()
    return seen


def waited(size, seed=1):
    s = Step(*size, seed)
    seen = steps_of(s, sync=True)
    torch.cuda.synchronize()
    assert s.B.device_error(clear=True) == 0
    return seen, [plan(ws)[1] for ws in s.ws[:2]]


def same(got, want):
    for a, b in zip(got, want, strict=True):
        assert torch.equal(a, b)


@pytest.mark.parametrize("size,pairs", [(PAIRS, 1), (PIECES, 1), (FEW, 0)], ids=["pairs", "pieces", "few"])
def test_results_do_not_depend_on_waiting_between_calls(size, pairs):
    want, ran = waited(size)
    assert ran == [pairs, pairs]
    for _ in range(3):
        s = Step(*size, 1)
        got = steps_of(s)
        torch.cuda.synchronize()
        assert s.B.device_error(clear=True) == 0
        same(got, want)


@pytest.mark.parametrize("sizes", [(PAIRS, PAIRS), (PAIRS, FEW), (PIECES, (600, 3000, 512, 1024))],
                         ids=["pairs", "pairs_and_few", "pairs_and_single"])
def test_two_streams_at_once(sizes):
    want = [waited(size, seed)[0] for size, seed in zip(sizes, (1, 2))]
    steps = [Step(*size, seed) for size, seed in zip(sizes, (1, 2))]
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
                s.update()
    torch.cuda.synchronize()
    assert steps[0].B.device_error(clear=True) == 0
    assert [plan(ws)[1] for ws in steps[0].ws[:2]] == [1, 1]
    for g, w in zip(got, want):
        same(g, w)


def test_graphs_with_one_workspace():
    """Three recorded calls, of which pairs take two, in the same workspace (each the part of
    it that it needs), replayed in turn."""
    steps = [Step(*PAIRS, 5), Step(*FEW, 6), Step(*PIECES, 7)]
    want, ran = [], []
    for s in steps:
        for call in s.calls():
            call()
        want.append(s.seen())
        ran.append([plan(ws)[1] for ws in s.ws[:2]])
    assert ran == [[1, 1], [0, 0], [1, 1]]
    torch.cuda.synchronize()
    shared = [max((s.ws[k] for s in steps), key=lambda w: w.numel()) for k in range(4)]
    graphs = []
    for s in steps:
        s.ws = [w[:own.numel()] for w, own in zip(shared, s.ws)]
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
        same(s.seen(), w)


def check(h, w, t, dl, loss, lse, dh, dw):
    """The comparison and the bounds of test_gpu_lmhead_loss.py, in fp64 on the GPU."""
    V, d = w.shape
    rows = torch.nonzero((t >= 0) & (t < V)).flatten()
    H, W, T, D, S = h[rows].double(), w.double(), t[rows].long(), dl[rows].double(), lse[rows].double()
    n, at = len(rows), torch.arange(len(rows), device=dev())
    off = torch.ones(len(h), dtype=torch.bool, device=dev())
    off[rows] = False
    assert not bool(loss[off].any()) and not bool(lse[off].any()) and not bool(dh[off].any())
    x = H @ W.T
    rs = torch.logsumexp(x, 1)
    rl = rs - x[at, T]
    ex = (d / 16 + 4) * STEP * (H.abs() @ W.abs().T).amax(1)
    size = torch.maximum(x.abs().amax(1), rs.abs())
    b = ex + 8 * U32 * size + 2.0 ** -21 + 64 * U32
    assert bool(((S - rs).abs() <= b + U32 * rs.abs()).all()), "lse"
    assert bool(((loss[rows].double() - rl).abs() <= 2 * b + 2 * U32 * (rl.abs() + size)).all()), "loss"
    p = torch.exp(x - S[:, None])
    hot = torch.zeros_like(p)
    hot[at, T] = 1.0
    g = (p - hot) * D[:, None]
    dg = p * D[:, None] * (ex + 8 * U32 * torch.maximum(size, S.abs()) + 2.0 ** -21)[:, None] + 2 * U32 * D[:, None] + 2.0 ** -8 * g.abs()
    mags = g.abs() + dg
    for got, want, b in ((dh[rows], g @ W, dg @ W.abs() + ((V / 16 + 4) * STEP + 65 * U32) * (mags @ W.abs())),
                         (dw, g.T @ H, dg.T @ H.abs() + (n / 16 + 8) * STEP * (mags.T @ H.abs()))):
        assert bool(((got.double() - want).abs() <= b + 2.0 ** -8 * (want.abs() + b) + 1e-40).all())


def test_a_captured_call_over_the_numbers_of_scored_rows_where_the_form_changes():
    """V d is large enough that the number of scored rows alone decides."""
    from paper_2608_02625_gb300 import binding as B
    N, V, d = 400, 62000, 2048
    g = torch.Generator(device=dev()).manual_seed(17)
    h = torch.empty(N, d, dtype=BF, device=dev()).normal_(generator=g)
    w = torch.empty(V, d, dtype=BF, device=dev()).normal_(0.0, d ** -0.5, generator=g)
    all_t = torch.randint(0, V, (N,), dtype=torch.int32, device=dev(), generator=g)
    dl = torch.rand(N, device=dev(), generator=g) + 0.25
    order = torch.randperm(N, device=dev(), generator=g)
    t = all_t.clone()
    new = lambda: [torch.empty(N, device=dev()), torch.empty(N, device=dev()), torch.empty_like(h), torch.empty_like(w)]  # noqa: E731
    ws = [torch.empty(k, dtype=torch.uint8, device=dev()) for k in (B.dlm_lmhead_loss_workspace_bytes(N, d),
                                                                  B.dlm_lmhead_loss_grad_workspace_bytes(N, V, d))]
    out = new()

    def go(o):
        B.dlm_lmhead_loss(h, w, t, o[0], o[1], ws[0])
        B.dlm_lmhead_loss_grad(h, w, t, o[1], dl, o[2], o[3], ws[1])

    go(out)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        go(out)
    for n in (400, 385, 384, 257, 256, 129, 128, 1, 0, 400):
        t.copy_(all_t)
        t[order[n:]] = -1
        direct = new()
        go(direct)
        for o in out:
            o.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert B.device_error(clear=True) == 0
        assert [plan(x) for x in ws] == [(n, int(n > 384 or 128 < n <= 256)), (n, int(n > 384))]
        same(out, direct)
        if n:
            check(h, w, t, dl, *out)
        else:
            assert not any(bool(o.any()) for o in out)


def test_two_host_threads_at_once():
    """Each with its own stream, buffers and size; the library's calls run without the
    interpreter's lock."""
    import threading
    sizes = [PAIRS, PIECES]
    want = [waited(size, seed)[0] for size, seed in zip(sizes, (1, 2))]
    steps = [Step(*size, seed) for size, seed in zip(sizes, (1, 2))]
    got, failed = [None, None], []
    torch.cuda.synchronize()

    def work(k):
        try:
            stream = torch.cuda.Stream(dev())
            with torch.cuda.device(dev()), torch.cuda.stream(stream):
                got[k] = steps_of(steps[k])
            stream.synchronize()
        except Exception as e:  # noqa: BLE001
            failed.append(e)

    threads = [threading.Thread(target=work, args=(k,)) for k in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed
    torch.cuda.synchronize()
    assert steps[0].B.device_error(clear=True) == 0
    for g, w in zip(got, want):
        same(g, w)
