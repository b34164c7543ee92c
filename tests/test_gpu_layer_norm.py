"""dlm_layer_norm and dlm_layer_norm_grad against the oracle in fp64.

Tolerances (U = 2^-24, half a step of fp32). A row's sums have at most 32 terms a
thread one after another (20 more in the widest rows), then 10 levels of pairs: a
relative error of at most 64 U of the sum of magnitudes, products and the division by
d included. So |mean| is off by 64 U mean|x|, rstd by 64 U relative (a wrong mean
enters the centred squares only in second order), xhat by both and a rounding of its
own, out by those times |w|, two roundings, and half a step of its type. The gradients
take mean and rstd as given."""
import numpy as np
import pytest
import torch

import oracle
from train_util import HALF, U32, Guarded, dev, host, within

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
SIZES = [(1, 1), (3, 7), (5, 8), (1, 64), (700, 64), (33, 100), (2, 200), (70, 1001), (9, 2048), (640, 2048), (301, 513),
         (5, 2501), (4, 4096), (3, 5001), (6, 8192), (4, 8191), (2, 8200), (3, 16384), (2, 20001)]
K = 64


def inputs(N, d, dt, wdt, seed=0):
    g = torch.Generator(device="cpu").manual_seed(seed + 1000 * N + d)
    x = torch.randn(N, d, generator=g) * 1.7 + torch.randn(d, generator=g) * 3.0 + 0.5
    x[:, ::97] *= 30.0
    return ((x.to(dt)).to(dev()), (1 + 0.3 * torch.randn(d, generator=g)).to(wdt).to(dev()),
            (0.3 * torch.randn(d, generator=g)).to(wdt).to(dev()), torch.randn(N, d, generator=g).to(dt).to(dev()))


def check_norm(x, w, b, out, mean, rstd, eps, where=""):
    X, W, Bv = host(x), host(w), 0.0 if b is None else host(b)
    ref, rm, rr = oracle.layer_norm(X, W, None if b is None else Bv, eps)
    dmean = K * U32 * np.abs(X).mean(1)
    if mean is not None:
        within(host(mean), rm, dmean + U32 * np.abs(rm), where + " mean")
    if rstd is not None:
        within(host(rstd), rr, K * U32 * rr, where + " rstd")
    xhat = (X - rm[:, None]) * rr[:, None]
    bound = np.abs(W) * (K * U32 * np.abs(xhat) + (dmean * rr)[:, None]) + 4 * U32 * (np.abs(W * xhat) + np.abs(Bv))
    within(host(out), ref, bound + HALF[x.dtype] * (np.abs(ref) + bound) + 1e-40, where + " out")


def check_grad(dy, x, w, mean, rstd, dx, dw, db, where=""):
    DY, X, W, M, R = (host(t) for t in (dy, x, w, mean, rstd))
    rx, rw, rb = oracle.layer_norm_grad(DY, X, W, M, R)
    N, d = X.shape
    xhat = (X - M[:, None]) * R[:, None]
    a = np.abs(DY * W)
    bound = K * U32 * R[:, None] * (a + a.mean(1)[:, None] + np.abs(xhat) * (a * np.abs(xhat)).mean(1)[:, None])
    within(host(dx), rx, bound + HALF[x.dtype] * (np.abs(rx) + bound) + 1e-40, where + " dx")
    # rows of one CTA one after another (at most N / 304 + 1), up to 32 groups of rows, 38 parts, 16 sums
    terms = N / 304 + 1 + 32 + 38 + 16 + 3
    for got, ref, mags in ((dw, rw, np.abs(DY * xhat).sum(0)), (db, rb, np.abs(DY).sum(0))):
        if got is not None:
            within(host(got), ref, terms * U32 * mags + HALF[got.dtype] * (np.abs(ref) + terms * U32 * mags) + 1e-40, where + " sums")


def run_grad(dy, x, w, mean, rstd, dx, dw, db):
    from paper_2608_02625_gb300 import binding as B
    ws = torch.full((B.dlm_layer_norm_grad_workspace_bytes(x.shape[:-1].numel(), x.shape[-1]),), 0xFF, dtype=torch.uint8, device=dev())
    B.dlm_layer_norm_grad(dy, x, w, mean, rstd, dx, dw, db, ws)


@pytest.mark.parametrize("dt,wdt", [(BF, BF), (BF, F32), (F32, F32), (F32, BF)])
@pytest.mark.parametrize("N,d", SIZES)
def test_norm_and_gradients(N, d, dt, wdt):
    from paper_2608_02625_gb300 import binding as B
    x, w, b, dy = inputs(N, d, dt, wdt)
    gd = Guarded()
    out, mean, rstd = gd.empty(N, d, dtype=dt), gd.empty(N), gd.empty(N)
    B.dlm_layer_norm(x, w, b, 1e-5, out, mean, rstd)
    gd.check()
    check_norm(x, w, b, out, mean, rstd, 1e-5, f"N={N} d={d}")
    dx, dw, db = gd.empty(N, d, dtype=dt), gd.empty(d, dtype=wdt), gd.empty(d, dtype=wdt)
    run_grad(dy, x, w, mean, rstd, dx, dw, db)
    gd.check()
    check_grad(dy, x, w, mean, rstd, dx, dw, db, f"N={N} d={d}")


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("N", [9, 1500])
@pytest.mark.parametrize("d", [768, 1280, 2560, 3080, 5120, 6144, 6152])
def test_widths_between_powers_of_two(N, d, dt):
    test_norm_and_gradients(N, d, dt, F32)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("d,row,offset", [(64, 80, 0), (64, 71, 0), (64, 64, 1), (2048, 2056, 8), (333, 400, 3), (8200, 8208, 8)])
def test_strided_rows_and_any_alignment(dt, d, row, offset):
    """Rows apart, in two leading dimensions, off 16-byte boundaries; no saved
    statistics, no bias; dweight or dbias alone."""
    from paper_2608_02625_gb300 import binding as B
    x, w, b, dy = inputs(6, d, dt, F32, seed=5)
    gd = Guarded()
    xs, dys = (gd.like(t.view(2, 3, d), offset=offset, row=row) for t in (x, dy))
    out = gd.empty(2, 3, d, dtype=dt, offset=offset, row=row)
    B.dlm_layer_norm(xs, w, None, 1e-3, out, None, None)
    gd.check()
    check_norm(x, w, None, out.reshape(6, d), None, None, 1e-3)
    mean, rstd = torch.empty(6, device=dev()), torch.empty(6, device=dev())
    B.dlm_layer_norm(xs, w, b, 1e-3, out, mean, rstd)
    for which in ((True, False), (False, True), (False, False)):
        dx = gd.empty(2, 3, d, dtype=dt, offset=offset, row=row)
        dw, db = (gd.empty(d) if on else None for on in which)
        if any(which):
            run_grad(dys, xs, w, mean, rstd, dx, dw, db)
        else:
            B.dlm_layer_norm_grad(dys, xs, w, mean, rstd, dx, None, None, None)
        gd.check()
        check_grad(dy, x, w, mean, rstd, dx.reshape(6, d), dw, db)


@pytest.mark.parametrize("d", [64, 2048, 8200])
def test_rows_of_one_value_and_large_means(d):
    """A constant row has variance 0; a mean 2^10 times the deviations keeps their accuracy."""
    from paper_2608_02625_gb300 import binding as B
    g = torch.Generator(device="cpu").manual_seed(d)
    x = torch.randn(5, d, generator=g)
    x[0] = 3.25
    x[1] += 1024.0
    x[2] *= 1e-6
    x = x.to(dev())
    w = torch.ones(d, device=dev())
    out, mean, rstd = torch.empty_like(x), torch.empty(5, device=dev()), torch.empty(5, device=dev())
    B.dlm_layer_norm(x, w, None, 1e-5, out, mean, rstd)
    torch.cuda.synchronize()
    check_norm(x, w, None, out, mean, rstd, 1e-5)


@pytest.mark.parametrize("d", [64, 2048, 8200])
def test_not_finite_rows_stay_alone(d):
    from paper_2608_02625_gb300 import binding as B
    x, w, b, _ = inputs(40, d, F32, F32, seed=2)
    clean = torch.empty_like(x)
    B.dlm_layer_norm(x, w, b, 1e-5, clean, None, None)
    x[3, 5], x[11, d - 1] = float("nan"), float("inf")
    out = torch.empty_like(x)
    B.dlm_layer_norm(x, w, b, 1e-5, out, None, None)
    bad = torch.zeros(40, dtype=torch.bool, device=dev())
    bad[3] = bad[11] = True
    assert bool(torch.isnan(out[bad]).all()) and torch.equal(out[~bad], clean[~bad])


def test_no_rows():
    from paper_2608_02625_gb300 import binding as B
    x = torch.empty(0, 64, device=dev())
    w = torch.ones(64, device=dev())
    none = torch.empty(0, device=dev())
    gd = Guarded()
    dw, db = gd.empty(64), gd.empty(64)
    B.dlm_layer_norm(x, w, None, 1e-5, torch.empty_like(x), none, none.clone())
    B.dlm_layer_norm_grad(torch.empty_like(x), x, w, none, none.clone(), torch.empty_like(x), dw, db, None)
    gd.check()
    assert bool((dw == 0).all()) and bool((db == 0).all())


def test_gradients_against_differences():
    """The gradients of sum(out * dy) against differences of the GPU's own norm in fp32:
    a step of 2^-5 in one element changes the sum by 2^-5 its gradient, within the sum's
    rounding and the step's third-order term."""
    from paper_2608_02625_gb300 import binding as B
    N, d, h = 3, 40, 2.0 ** -5
    x, w, b, dy = inputs(N, d, F32, F32, seed=8)
    x = x / 8

    def value(x, w, b):
        out = torch.empty_like(x)
        B.dlm_layer_norm(x, w, b, 1e-5, out, None, None)
        return float((out.double() * dy.double()).sum())

    out, mean, rstd = torch.empty_like(x), torch.empty(N, device=dev()), torch.empty(N, device=dev())
    B.dlm_layer_norm(x, w, b, 1e-5, out, mean, rstd)
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)
    run_grad(dy, x, w, mean, rstd, dx, dw, db)
    size = float((out.abs().double() * dy.abs().double()).sum())
    # third derivatives of xhat in one element are below 15 rstd^3 |dy| per element of the row
    r = host(rstd)
    curve = 15 * h * h / 6 * (r ** 3)[:, None] * np.abs(host(dy * w)).sum(1)[:, None]
    noise = 8 * K * U32 * size / (2 * h)
    for t, grad, extra in ((x, dx, np.broadcast_to(curve, x.shape)), (w, dw, np.zeros(d)), (b, db, np.zeros(d))):
        flat, gflat, ex = t.view(-1), host(grad).reshape(-1), extra.reshape(-1)
        for i in range(0, flat.numel(), 7):
            old = flat[i].item()
            flat[i] = old + h
            up = value(x, w, b)
            flat[i] = old - h
            down = value(x, w, b)
            flat[i] = old
            assert abs((up - down) / (2 * h) - gflat[i]) <= noise + ex[i]


def test_same_bits_again_and_on_another_stream_and_replayed():
    from paper_2608_02625_gb300 import binding as B
    x, w, b, dy = inputs(700, 2048, BF, F32, seed=3)
    new = lambda: [torch.empty_like(x), torch.empty(700, device=dev()), torch.empty(700, device=dev()),  # noqa: E731
                   torch.empty_like(x), torch.empty_like(w), torch.empty_like(w)]
    ws = torch.empty(B.dlm_layer_norm_grad_workspace_bytes(700, 2048), dtype=torch.uint8, device=dev())

    def go(o, ws):
        B.dlm_layer_norm(x, w, b, 1e-5, o[0], o[1], o[2])
        B.dlm_layer_norm_grad(dy, x, w, o[1], o[2], o[3], o[4], o[5], ws)

    first = new()
    go(first, ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    second = new()
    with torch.cuda.stream(side):
        go(second, torch.empty_like(ws))
    side.synchronize()
    third = new()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        go(third, ws)
    for t in third:
        t.fill_(0)
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    for a, b_, c in zip(first, second, third):
        assert torch.equal(a, b_) and torch.equal(a, c)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("d", [64, 1001, 2048, 5120, 8191, 8200])
def test_gradients_of_rows_of_tiny_deviations(d, dt):
    """eps = 0 and deviations of 1e-20: rstd is 1e20, whose square fp32 does not hold, the
    gradients are of that size."""
    _, w, _, dy = inputs(9, d, dt, F32, seed=9)
    x = (torch.randn(9, d, generator=torch.Generator(device="cpu").manual_seed(d)) * 1e-20).to(dt).to(dev())
    mean, rstd = (torch.from_numpy(v).float().to(dev()) for v in oracle.layer_norm(host(x), host(w), None, 0.0)[1:])
    gd = Guarded()
    dx, dw, db = gd.empty(9, d, dtype=dt), gd.empty(d), gd.empty(d)
    run_grad(dy, x, w, mean, rstd, dx, dw, db)
    gd.check()
    check_grad(dy, x, w, mean, rstd, dx, dw, db, f"d={d}")


def test_offsets_past_32_bits():
    """2.3e9 elements: the first and the last rows, and the sums over the columns, against
    fp64 on the GPU. (Sums of ones times x: dbias is the number of rows exactly.)"""
    from paper_2608_02625_gb300 import binding as B
    N, d = 1_130_000, 2048
    g = torch.Generator(device=dev()).manual_seed(4)
    x = torch.empty(N, d, dtype=BF, device=dev()).normal_(generator=g)
    w, b = 1 + 0.3 * torch.randn(d, device=dev(), generator=g), torch.randn(d, device=dev(), generator=g)
    out, mean, rstd = torch.empty_like(x), torch.empty(N, device=dev()), torch.empty(N, device=dev())
    B.dlm_layer_norm(x, w, b, 1e-5, out, mean, rstd)
    dy, dx, dw, db = torch.ones_like(x), torch.empty_like(x), torch.empty(d, device=dev()), torch.empty(d, device=dev())
    run_grad(dy, x, w, mean, rstd, dx, dw, db)
    for r in (slice(0, 3), slice(2 ** 31 // d - 1, 2 ** 31 // d + 2), slice(N - 3, N)):
        check_norm(x[r], w, b, out[r], mean[r], rstd[r], 1e-5)
        check_grad(dy[r], x[r], w, mean[r], rstd[r], dx[r], None, None)
    assert bool((db == N).all())
    want, mags = torch.zeros(d, dtype=torch.float64, device=dev()), torch.zeros(d, dtype=torch.float64, device=dev())
    for i in range(0, N, 50_000):
        xhat = (x[i:i + 50_000].double() - mean[i:i + 50_000, None].double()) * rstd[i:i + 50_000, None].double()
        want += xhat.sum(0)
        mags += xhat.abs().sum(0)
    # rows of one group one after another (N / 608 at most), then as in check_grad
    assert bool(((dw.double() - want).abs() <= (N / 608 + 1 + 89) * U32 * mags).all())
