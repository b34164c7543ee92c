"""The projection loss and its gradients where CTAs work in pairs: calls that follow each
other without a wait, two streams at once, and graphs that share a workspace. What ran is
read from the start of the workspace (the scored rows, and whether pairs took them), so that
a later rule for the choice cannot take the pairs out of these tests unseen."""
import pytest
import torch

from test_gpu_train_overlap import Step
from train_util import dev

pytestmark = pytest.mark.gpu

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
