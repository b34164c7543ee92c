"""dlm_clip_grad_norm against the oracle in fp64.

Tolerances: a thread adds at most 32 squares one after another in each of eight fp32
sums and three levels of pairs, everything else in fp64: the sum of squares is off by
at most 37 U relative (U = 2^-24), the norm by half of that and its own rounding, 20 U;
an output by the norm's 20 U, the factor's and the product's roundings, and half a step
of its type. Below 2^-126 fp32's steps are 2^-149 whatever the value, so a rounding there
is off by up to 2^-150, absolute."""
import numpy as np
import pytest
import torch

import oracle
from train_util import HALF, U32, Guarded, dev, host, within

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def workspace():
    from paper_2608_02625_gb300 import binding as B
    return torch.full((B.dlm_clip_grad_norm_workspace_bytes(),), 0xFF, dtype=torch.uint8, device=dev())


def make(sizes, dtypes, seed=0, std=1e-3):
    g = torch.Generator(device="cpu").manual_seed(seed)
    return [(torch.randn(n, generator=g) * std).to(dtypes[i % len(dtypes)]).to(dev()) for i, n in enumerate(sizes)]


def check(grads, outs, norm, max_norm, where=""):
    ref, n = oracle.clip_grad_norm([host(g) for g in grads], max_norm)
    within(host(norm), [n], 20 * U32 * n + 2.0 ** -150, where + " norm")
    for i, (o, r) in enumerate(zip(outs or (), ref)):
        within(host(o), r, (24 * U32 + HALF[o.dtype]) * np.abs(r) + 2.0 ** -149, f"{where} tensor {i}")


CASES = {
    "one": ([1], [F32]), "one_odd_bf16": ([7], [BF]), "chunk_edges": ([2047, 2048, 2049, 4096, 1], [F32, BF]),
    "empty_ones": ([0, 5, 0, 0, 300, 0], [BF]), "all_empty": ([0, 0], [F32]),
    "long": ([3_000_001], [BF]), "long_f32": ([1_000_000, 17], [F32]), "head": ([2_000_000, 2048, 2048], [BF, F32]),
    "seventeen": ([100 + i for i in range(17)], [F32, BF]), "many": ([1 + (i * 37) % 400 for i in range(129)], [BF, F32]),
    "two_launches": ([1 + (i * 13) % 50 for i in range(1100)], [F32, BF]),
}


@pytest.mark.parametrize("name", CASES)
@pytest.mark.parametrize("share", [0.3, 1.5, float("inf"), 0.0])
def test_norm_and_outputs(name, share):
    from paper_2608_02625_gb300 import binding as B
    grads = make(*CASES[name])
    full = oracle.clip_grad_norm([host(g) for g in grads], 1.0)[1]
    max_norm = share * full if full else share
    gd = Guarded()
    outs, norm = [gd.empty(*g.shape, dtype=g.dtype) for g in grads], gd.empty(1)
    B.dlm_clip_grad_norm(grads, outs, max_norm, norm, workspace())
    gd.check()
    check(grads, outs, norm, np.float64(np.float32(max_norm)), name)
    if share > 1:
        assert all(torch.equal(g, o) for g, o in zip(grads, outs))


@pytest.mark.parametrize("share", [0.3, 1.5])
def test_in_place_tuple_and_norm_alone(share):
    from paper_2608_02625_gb300 import binding as B
    grads = make([5000, 3, 0, 70000], [BF, F32], seed=2)
    before = [g.clone() for g in grads]
    n = oracle.clip_grad_norm([host(g) for g in grads], 1.0)[1]
    norm = torch.empty(1, device=dev())
    B.dlm_clip_grad_norm(tuple(grads), None, share * n, norm, workspace())
    check(before, None, norm, share * n)
    assert all(torch.equal(a, b) for a, b in zip(before, grads))
    B.dlm_clip_grad_norm(grads, grads, share * n, norm, workspace())
    check(before, grads, norm, np.float64(np.float32(share * n)))


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("offset", [1, 3, 8])
def test_any_alignment_and_rank(dt, offset):
    from paper_2608_02625_gb300 import binding as B
    grads = [g.to(dt) for g in make([60, 5001, 2048], [F32], seed=offset)]
    gd = Guarded()
    shapes = [(3, 4, 5, 1), (5001,), (32, 64)]
    views = [gd.like(g.view(s), offset=offset) for g, s in zip(grads, shapes)]
    outs, norm = [gd.empty(*s, dtype=dt, offset=(offset + 1) % 4) for s in shapes], gd.empty(1, offset=1)
    B.dlm_clip_grad_norm(views, outs, 0.01, norm, workspace())
    gd.check()
    check(grads, [o.reshape(-1) for o in outs], norm, np.float64(np.float32(0.01)))


@pytest.mark.parametrize("value", [1e30, 3e38, 1e-25, 1e-38, 1e-42])
def test_values_whose_squares_leave_the_range(value):
    """Beside ordinary chunks of zeros; the factor itself below fp32's normal range too."""
    from paper_2608_02625_gb300 import binding as B
    g = torch.zeros(200_000, device=dev())
    g[::7] = value
    g[1] = -value
    grads = [g, torch.zeros(5000, dtype=BF, device=dev())]
    n = oracle.clip_grad_norm([host(t) for t in grads], 1.0)[1]
    outs, norm = [torch.empty_like(t) for t in grads], torch.empty(1, device=dev())
    B.dlm_clip_grad_norm(grads, outs, 1e-3, norm, workspace())
    if n > 3.4028235e38:  # the norm itself is above fp32's largest number
        assert float(norm) == float("inf")
        ref = oracle.clip_grad_norm([host(t) for t in grads], np.float64(np.float32(1e-3)))[0]
        for o, r in zip(outs, ref):
            within(host(o), r, 26 * U32 * np.abs(r) + 2.0 ** -149)
    else:
        check(grads, outs, norm, np.float64(np.float32(1e-3)), f"{value}")


def test_not_finite():
    from paper_2608_02625_gb300 import binding as B
    for bad in (float("nan"), float("inf")):
        grads = make([5000, 40], [BF, F32], seed=4)
        grads[0][77] = bad
        outs, norm = [torch.empty_like(g) for g in grads], torch.empty(1, device=dev())
        B.dlm_clip_grad_norm(grads, outs, 1.0, norm, workspace())
        if bad != bad:
            assert bool(torch.isnan(norm).all()) and all(bool(torch.isnan(o).all()) for o in outs)
        else:
            assert float(norm) == bad and bool(torch.isnan(outs[0][77])) and bool((outs[1] == 0).all())
            assert int(torch.isnan(outs[0]).sum()) == 1


def test_an_infinity_under_an_infinite_limit():
    from paper_2608_02625_gb300 import binding as B
    grads = make([5000, 40], [BF, F32], seed=4)
    grads[0][77] = float("inf")
    outs, norm = [torch.empty_like(g) for g in grads], torch.empty(1, device=dev())
    B.dlm_clip_grad_norm(grads, outs, float("inf"), norm, workspace())
    assert float(norm) == float("inf") and all(bool(torch.isnan(o).all()) for o in outs)


def test_no_tensors():
    from paper_2608_02625_gb300 import binding as B
    for outs in (None, []):
        norm = torch.full((1,), -1.0, device=dev())
        B.dlm_clip_grad_norm([], outs, 1.0, norm, workspace())
        assert float(norm) == 0.0


def test_same_bits_again_on_another_stream_and_replayed():
    from paper_2608_02625_gb300 import binding as B
    grads = make([1_500_000, 2048, 2047, 3], [BF, F32], seed=6)
    new = lambda: [torch.empty_like(g) for g in grads] + [torch.empty(1, device=dev())]  # noqa: E731
    ws = workspace()
    first, second, third = new(), new(), new()
    B.dlm_clip_grad_norm(grads, first[:-1], 0.5, first[-1], ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        B.dlm_clip_grad_norm(grads, second[:-1], 0.5, second[-1], workspace())
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        B.dlm_clip_grad_norm(grads, third[:-1], 0.5, third[-1], ws)
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    for a, b, c in zip(first, second, third):
        assert torch.equal(a, b) and torch.equal(a, c)


@pytest.mark.parametrize("dt,offset,big", [(F32, 0, 1024), (F32, 1, 256), (BF, 0, 2048), (BF, 1, 256)])
def test_small_squares_behind_a_large_one(dt, offset, big):
    """Chunks of 32768 elements (from 75 M in all), 128 a thread, of which each thread's first
    ones are 4096 and the others 0.98: beside 2^24 a square below 1 is lost. In eight sums of
    at most 17 squares, three levels of pairs and fp64 beyond them the sum of squares is off by
    20 U relative at most, the norm by half of that and its own rounding; one sum of 128 loses
    62 U of the norm here, four of 32 15 U."""
    from paper_2608_02625_gb300 import binding as B
    n = 80_000_003
    x = torch.full((n + offset,), 0.98, dtype=dt, device=dev())[offset:]
    x[torch.arange(n, device=dev()) % 32768 < big] = 4096.0
    want = float(sum(p.double().square().sum() for p in x.split(10_000_000)) ** 0.5)
    norm = torch.empty(1, device=dev())
    B.dlm_clip_grad_norm([x], None, 1.0, norm, workspace())
    assert abs(float(norm) - want) <= 12 * U32 * want


def test_offsets_past_32_bits():
    """2.2e9 elements behind a small tensor, in place."""
    from paper_2608_02625_gb300 import binding as B
    n = 2_200_000_007
    x = torch.full((n,), 2.0 ** -6, dtype=BF, device=dev())
    x[-5:] = 3.0
    small = torch.full((77,), 0.5, device=dev())
    want = (n * 2.0 ** -12 + 5 * (9.0 - 2.0 ** -12) + 77 * 0.25) ** 0.5
    norm = torch.empty(1, device=dev())
    B.dlm_clip_grad_norm([small, x], [small, x], want / 2, norm, workspace())
    assert abs(float(norm) - want) <= 12 * U32 * want
    # the factor is 1/2 but for 1e-6 / norm and the norm's roundings, lost in bf16's
    assert bool((x[:-5] == 2.0 ** -7).all()) and bool((x[-5:] == 1.5).all())
    assert float((small - 0.25).abs().max()) <= 0.25 * (16 * U32 + 1e-6 / want)


def test_empty_gradients_of_several_dimensions():
    from paper_2608_02625_gb300 import binding as B
    grads = make([500], [F32], seed=9) + [torch.empty(s, dtype=BF, device=dev()) for s in ((5, 0), (0, 7), (2, 0, 3))]
    outs, norm = [torch.empty_like(g) for g in grads], torch.empty(1, device=dev())
    B.dlm_clip_grad_norm(grads, outs, 1e-3, norm, workspace())
    check(grads[:1], outs[:1], norm, np.float64(np.float32(1e-3)))
