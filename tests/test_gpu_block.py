"""dlm_gated_linear, dlm_linear and their gradients against the oracle in fp64 (tolerances:
block_util)."""
import numpy as np
import pytest
import torch

import oracle
from block_util import (ACTS, BF, F32, Guarded, check_gated, check_gated_grad, check_linear, check_linear_grad, dev, host, rand,
                        workspace)

pytestmark = pytest.mark.gpu

# rows, width, inner width
SIZES = [(1, 8, 8), (3, 8, 16), (1, 64, 264), (2, 2048, 520), (7, 72, 1000), (16, 4096, 64), (17, 200, 136), (33, 512, 2048),
         (64, 512, 1032), (65, 64, 304), (100, 1032, 128), (128, 64, 128), (129, 200, 264), (130, 72, 1000), (257, 320, 1024),
         (300, 128, 2048), (517, 200, 1000), (700, 1024, 600), (1000, 264, 520), (2100, 64, 304)]


def block(N, d, f, seed=0):
    return (rand(N, d, seed=seed + N), rand(f, d, seed=seed + 1, std=d ** -0.5), rand(f, d, seed=seed + 2, std=d ** -0.5))


def grad_ws(N, f, d, gd=None):
    from paper_2608_02625_gb300 import binding as B
    return workspace(B.dlm_gated_linear_grad_workspace_bytes, N, f, d, gd=gd)


def linear_ws(N, m, k, gd=None):
    from paper_2608_02625_gb300 import binding as B
    return workspace(B.dlm_linear_workspace_bytes, N, m, k, gd=gd)


def linear_grad_ws(N, m, k, gd=None):
    from paper_2608_02625_gb300 import binding as B
    return workspace(B.dlm_linear_grad_workspace_bytes, N, m, k, gd=gd)


def no_error():
    from paper_2608_02625_gb300 import binding as B
    assert B.device_error(clear=True) == 0


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("keep", [False, True], ids=["", "keep"])
@pytest.mark.parametrize("N,d,f", SIZES)
def test_gated(N, d, f, keep, act):
    from paper_2608_02625_gb300 import binding as B
    x, wg, wu = block(N, d, f)
    gd = Guarded()
    out = gd.empty(N, f, dtype=BF, row=f + 8)
    gate, up = (gd.empty(N, f, dtype=BF), gd.empty(N, f, dtype=BF, row=f + 24)) if keep else (None, None)
    B.dlm_gated_linear(x, wg, wu, ACTS[act], out, gate, up)
    gd.check()
    check_gated(x, wg, wu, act, out, gate, up)
    no_error()


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("add", ["no", "other", "itself"])
@pytest.mark.parametrize("N,d,f", SIZES)
def test_gated_grad(N, d, f, add, act):
    from paper_2608_02625_gb300 import binding as B
    x, wg, wu = block(N, d, f)
    gate, up = (x.float() @ wg.float().T).to(BF), (x.float() @ wu.float().T).to(BF)
    dout = rand(N, f, seed=5)
    gd = Guarded()
    dx, dwg, dwu = gd.empty(N, d, dtype=BF, row=d + 3, offset=1), gd.empty(f, d, dtype=BF, row=d + 8), gd.empty(f, d, dtype=BF)
    extra, given = None, None
    if add == "other":
        given = extra = gd.like(rand(N, d, seed=6), row=d + 1, offset=3)
    if add == "itself":
        dx.copy_(rand(N, d, seed=6))
        given, extra = dx, dx.clone()
    ws = grad_ws(N, f, d, gd)
    B.dlm_gated_linear_grad(dout, x, wg, wu, gate, up, ACTS[act], given, dx, dwg, dwu, ws)
    gd.check()
    check_gated_grad(dout, x, wg, wu, gate, up, act, extra, dx, dwg, dwu)
    no_error()


@pytest.mark.parametrize("act,bias,residual,keep", [("none", None, "no", False), ("silu", BF, "other", True), ("gelu", F32, "itself", True),
                                                   ("none", F32, "other", True), ("gelu", None, "no", True), ("silu", F32, "itself", False)])
@pytest.mark.parametrize("N,k,m", SIZES + [(n, b, a) for n, a, b in SIZES])
def test_linear(N, k, m, act, bias, residual, keep):
    from paper_2608_02625_gb300 import binding as B
    x, w = rand(N, k, seed=N), rand(m, k, seed=1, std=k ** -0.5)
    gd = Guarded()
    b = None if bias is None else gd.like(rand(m, seed=2, std=0.5, dtype=bias), offset=1)
    out = gd.empty(N, m, dtype=BF, row=m + 5, offset=3)
    given, r = None, None
    if residual == "other":
        given = r = gd.like(rand(N, m, seed=3), row=m + 1, offset=5)
    if residual == "itself":
        out.copy_(rand(N, m, seed=3))
        given, r = out, out.clone()
    pre = gd.empty(N, m, dtype=BF, row=m + 7, offset=1) if keep else None
    B.dlm_linear(x, w, b, ACTS[act], given, out, pre, linear_ws(N, m, k, gd))
    gd.check()
    check_linear(x, w, b, act, r, out, pre)
    no_error()


@pytest.mark.parametrize("act,bias,add", [("none", None, "no"), ("silu", BF, "other"), ("gelu", F32, "itself"), ("none", F32, "other")])
@pytest.mark.parametrize("N,k,m", SIZES + [(n, b, a) for n, a, b in SIZES])
def test_linear_grad(N, k, m, act, bias, add):
    from paper_2608_02625_gb300 import binding as B
    x, w, dout = rand(N, k, seed=N), rand(m, k, seed=1, std=k ** -0.5), rand(N, m, seed=5)
    gd = Guarded()
    pre = None if act == "none" else gd.like(rand(N, m, seed=4, std=2.0), row=m + 8)
    dx, dw = gd.empty(N, k, dtype=BF, row=k + 9, offset=1), gd.empty(m, k, dtype=BF, row=k + 8)
    db = None if bias is None else gd.empty(m, dtype=bias, offset=1)
    given, extra = None, None
    if add == "other":
        given = extra = gd.like(rand(N, k, seed=6), row=k + 1, offset=3)
    if add == "itself":
        dx.copy_(rand(N, k, seed=6))
        given, extra = dx, dx.clone()
    B.dlm_linear_grad(dout, x, w, pre, ACTS[act], given, dx, dw, db, linear_grad_ws(N, m, k, gd))
    gd.check()
    check_linear_grad(dout, x, w, pre, act, extra, dx, dw, db)
    no_error()


@pytest.mark.parametrize("N", [40, 300])
def test_parts_of_the_gradients(N):
    """Each result alone has the bits that it has beside the others."""
    from paper_2608_02625_gb300 import binding as B
    d, f = 136, 520
    x, wg, wu = block(N, d, f)
    dout, gate, up, pre = (rand(N, f, seed=s) for s in (5, 6, 7, 8))
    e = lambda *s, t=BF: torch.empty(*s, dtype=t, device=dev())  # noqa: E731
    ws = grad_ws(N, f, d)
    dx, dwg, dwu = e(N, d), e(f, d), e(f, d)
    B.dlm_gated_linear_grad(dout, x, wg, wu, gate, up, 1, None, dx, dwg, dwu, ws)
    one, two, three = e(N, d), e(f, d), e(f, d)
    B.dlm_gated_linear_grad(dout, x, wg, wu, gate, up, 1, None, one, None, None, ws)
    B.dlm_gated_linear_grad(dout, x, wg, wu, gate, up, 1, None, None, two, three, ws)
    assert torch.equal(dx, one) and torch.equal(dwg, two) and torch.equal(dwu, three)
    ws = linear_grad_ws(N, f, d)
    db = e(f, t=F32)
    B.dlm_linear_grad(dout, x, wg, pre, 1, None, dx, dwg, db, ws)
    one, two, three = e(N, d), e(f, d), e(f, t=F32)
    B.dlm_linear_grad(dout, x, wg, pre, 1, None, one, None, None, ws)
    B.dlm_linear_grad(dout, x, wg, pre, 1, None, None, two, None, ws)
    B.dlm_linear_grad(dout, x, wg, pre, 1, None, None, None, three, ws)
    assert torch.equal(dx, one) and torch.equal(dwg, two) and torch.equal(db, three)
    B.dlm_linear_grad(dout, x, wg, None, 0, None, None, None, db, ws)
    check_linear_grad(dout, x, wg, None, "none", None, None, None, db)


@pytest.mark.parametrize("L", [1, 5, 90])
def test_batches_and_strided_rows(L):
    """[B, L, d] inputs that are parts of a packed tensor, and one that a slice leaves."""
    from paper_2608_02625_gb300 import binding as B
    packed = rand(3, L, 3 * 64 + 8, seed=1)
    x = packed[..., 64:128]
    wg, wu = rand(136, 80, seed=2, std=0.1)[:, 8:72], rand(136, 64, seed=3, std=0.1)
    out = torch.zeros(3, L, 2 * 136, dtype=BF, device=dev())
    B.dlm_gated_linear(x, wg, wu, 2, out[..., 136:], None, None)
    check_gated(x, wg, wu, "gelu", out[..., 136:])
    assert not out[..., :136].any()
    y = torch.zeros(3, L, 2 * 64 + 1, dtype=BF, device=dev())
    B.dlm_linear(out[..., 136:], rand(64, 136, seed=4, std=0.1), None, 0, x, y[..., 1:65], None, linear_ws(3 * L, 64, 136))
    check_linear(out[..., 136:], rand(64, 136, seed=4, std=0.1), None, "none", x, y[..., 1:65])
    assert not y[..., 0].any() and not y[..., 65:].any()


@pytest.mark.parametrize("N", [1, 20, 300])
def test_column_ranges_of_one_buffer(N):
    """Tensors whose rows lie between each other's: the same bits as apart, and nothing else written."""
    from paper_2608_02625_gb300 import binding as B
    d, f = 136, 264
    x, wg, wu = block(N, d, f)
    e = lambda *s: torch.full(s, 7.0, dtype=BF, device=dev())  # noqa: E731
    wide, apart = e(N, 3 * f + 16), [e(N, f) for _ in range(3)]
    parts = [wide[:, i * (f + 8):i * (f + 8) + f] for i in range(3)]
    for out, gate, up in (parts, apart):
        B.dlm_gated_linear(x, wg, wu, 1, out, gate, up)
    assert all(torch.equal(a, b) for a, b in zip(parts, apart))
    assert bool((wide[:, f:f + 8] == 7).all()) and bool((wide[:, 2 * f + 8:2 * f + 16] == 7).all())
    # weights beside their gradients, dx beside x
    w = e(f, 4 * d)
    ws, dws = (w[:, :d], w[:, d:2 * d]), (w[:, 2 * d:3 * d], w[:, 3 * d:])
    for to, t in zip(ws, (wg, wu)):
        to.copy_(t)
    xs = e(N, 2 * d)
    xs[:, :d].copy_(x)
    dout = rand(N, f, seed=3)
    dx, dw = e(N, d), [e(f, d) for _ in range(2)]
    B.dlm_gated_linear_grad(dout, x, wg, wu, apart[1], apart[2], 1, x, dx, *dw, grad_ws(N, f, d))
    B.dlm_gated_linear_grad(dout, xs[:, :d], *ws, parts[1], parts[2], 1, xs[:, :d], xs[:, d:], *dws, grad_ws(N, f, d))
    assert torch.equal(xs[:, d:], dx) and torch.equal(xs[:, :d], x) and all(torch.equal(a, b) for a, b in zip(dws, dw))
    assert torch.equal(ws[0], wg) and torch.equal(ws[1], wu)
    # a projection's result and its pre beside the residual
    for r in (parts, apart):
        r[2].copy_(dout)
        B.dlm_linear(x, wg, None, 2, r[2], r[0], r[1], linear_ws(N, f, d))
    assert all(torch.equal(a, b) for a, b in zip(parts, apart)) and torch.equal(parts[2], dout)
    B.dlm_linear_grad(dout, x, wg, apart[1], 2, None, dx, dw[0], None, linear_grad_ws(N, f, d))
    B.dlm_linear_grad(dout, xs[:, :d], ws[0], parts[1], 2, None, xs[:, d:], dws[0], None, linear_grad_ws(N, f, d))
    assert torch.equal(xs[:, d:], dx) and torch.equal(dws[0], dw[0]) and torch.equal(xs[:, :d], x)
    no_error()


@pytest.mark.parametrize("N", [5, 100, 400])
def test_what_is_not_part_of_a_tensor_is_not_read(N):
    """NaN around every input: behind the last row and between rows."""
    from paper_2608_02625_gb300 import binding as B
    d, f = 72, 200

    def within_nan(t):
        buf = torch.full((t.shape[0] + 300, t.shape[1] + 16), float("nan"), dtype=BF, device=dev())
        view = buf[:t.shape[0], :t.shape[1]]
        view.copy_(t)
        return view

    x, wg, wu = map(within_nan, block(N, d, f))
    gate, up, out, dout = (within_nan(rand(N, f, seed=s)) for s in range(4))
    B.dlm_gated_linear(x, wg, wu, 1, out, gate, up)
    check_gated(x, wg, wu, "silu", out, gate, up)
    dx, dwg, dwu = torch.empty(N, d, dtype=BF, device=dev()), torch.empty(f, d, dtype=BF, device=dev()), torch.empty(f, d, dtype=BF, device=dev())
    B.dlm_gated_linear_grad(dout, x, wg, wu, gate, up, 1, None, dx, dwg, dwu, grad_ws(N, f, d))
    check_gated_grad(dout, x, wg, wu, gate, up, "silu", None, dx, dwg, dwu)
    for act, pre in (("none", None), ("gelu", gate)):
        B.dlm_linear_grad(dout, x, wg, pre, ACTS[act], None, dx, dwg, None, linear_grad_ws(N, f, d))
        check_linear_grad(dout, x, wg, pre, act, None, dx, dwg, None)
    y = torch.empty(N, f, dtype=BF, device=dev())
    B.dlm_linear(x, wg, None, 0, None, y, None, linear_ws(N, f, d))
    check_linear(x, wg, None, "none", None, y)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("N", [6, 150, 300])
def test_bad_rows_stay_alone(N, bad):
    from paper_2608_02625_gb300 import binding as B
    x, wg, wu = block(N, 128, 264)
    x[4, 7] = bad
    out, gate, up = (torch.empty(N, 264, dtype=BF, device=dev()) for _ in range(3))
    B.dlm_gated_linear(x, wg, wu, 1, out, gate, up)
    y = torch.empty(N, 264, dtype=BF, device=dev())
    B.dlm_linear(x, wg, None, 2, None, y, None, linear_ws(N, 264, 128))
    rest = torch.arange(N, device=dev()) != 4
    for t in (out, gate, up, y):
        assert bool(torch.isfinite(t[rest]).all())
    assert not bool(torch.isfinite(gate[4]).any())


def test_activations_far_out():
    """Products of any size: where act and its slope have long reached their ends."""
    from paper_2608_02625_gb300 import binding as B
    z = torch.tensor([0.0, 1e-30, 1.0, 3.0, 9.0, 20.0, 80.0, 99.0, 101.0, 300.0, 1e4, 1e10, 1e20, 3e38], device=dev()).to(BF)
    z = torch.cat([z, -z, torch.tensor([float("nan"), float("inf")], device=dev()).to(BF)])
    z = torch.cat([z, torch.zeros(32 - len(z), dtype=BF, device=dev())])
    eye = torch.eye(32, dtype=BF, device=dev())
    ones = torch.ones(32, 32, dtype=BF, device=dev())
    for act in ("silu", "gelu"):
        for N in (1, 300):
            gate, up, dout = z.repeat(N, 1), torch.ones(N, 32, dtype=BF, device=dev()), torch.ones(N, 32, dtype=BF, device=dev())
            dx, db = torch.empty(N, 32, dtype=BF, device=dev()), torch.empty(32, device=dev())
            value, slope = (torch.from_numpy(t) for t in oracle.activation(act, host(z[:-4])))
            finite = torch.arange(28)
            # dbias of one row is that row's dz, in fp32
            B.dlm_linear_grad(dout[:1], dx[:1].fill_(1.0), eye, gate[:1], ACTS[act], None, None, None, db, linear_grad_ws(1, 32, 32))
            got = db.double().cpu()[finite]
            far = host(z[:28]).__abs__() > 100.0
            want = torch.where(torch.from_numpy(far), (torch.from_numpy(host(z[:28])) > 0).double(), slope[finite])
            assert float((got - want).abs().max()) <= 2e-5, (act, got, want)
            assert bool(torch.isnan(db[28])) and float(db[29]) == 1.0
            # the value, as dup of a gate given
            dwu = torch.empty(32, 32, dtype=BF, device=dev())
            B.dlm_gated_linear_grad(dout[:1], ones[:1], eye, eye, gate[:1], up[:1], ACTS[act], None, None, torch.empty_like(dwu), dwu,
                                    grad_ws(1, 32, 32))
            v = dwu[:28, 0].double().cpu()
            np.testing.assert_allclose(v.numpy(), np.where(far, np.maximum(host(z[:28]), 0.0), value[finite].numpy()), rtol=2.0 ** -7, atol=1e-30)


def test_gradients_of_no_rows():
    from paper_2608_02625_gb300 import binding as B
    e = lambda *s, t=BF: torch.full(s, 7.0, dtype=t, device=dev())  # noqa: E731
    dwg, dwu, db = e(40, 80)[:, :64], e(40, 64), e(40, t=F32)
    none, wide = e(0, 40), e(0, 64)
    B.dlm_gated_linear_grad(none, wide, e(40, 64), e(40, 64), none, none, 1, None, wide, dwg, dwu, e(1, t=F32))
    assert not dwg.any() and not dwu.any()
    dwg.fill_(1)
    B.dlm_linear_grad(none, wide, e(40, 64), none, 1, None, wide, dwg, db, e(1, t=F32))
    assert not dwg.any() and not db.any()
    B.dlm_gated_linear(wide, dwg, dwu, 1, none, None, None)
    B.dlm_linear(wide, dwg, db, 1, None, none, None, None)


@pytest.mark.parametrize("N,d,f", [(9, 200, 1000), (700, 264, 600), (1500, 2048, 256), (300, 64, 6000)])
def test_the_same_bits_every_time(N, d, f):
    from paper_2608_02625_gb300 import binding as B
    x, wg, wu = block(N, d, f)
    dout, gate, up, bias = rand(N, f, seed=1), rand(N, f, seed=2), rand(N, f, seed=3), rand(f, seed=4, dtype=F32)
    first = None
    for _ in range(4):
        e = [torch.empty(*s, dtype=BF, device=dev()) for s in ((N, f), (N, f), (N, d), (f, d), (f, d), (N, d), (f, d))]
        db = torch.empty(f, device=dev())
        B.dlm_gated_linear(x, wg, wu, 1, e[0], None, None)
        B.dlm_linear(x, wg, bias, 2, None, e[1], None, linear_ws(N, f, d))
        B.dlm_gated_linear_grad(dout, x, wg, wu, gate, up, 1, None, e[2], e[3], e[4], grad_ws(N, f, d))
        B.dlm_linear_grad(dout, x, wg, gate, 2, None, e[5], e[6], db, linear_grad_ws(N, f, d))
        first = first or [t.clone() for t in e + [db]]
        assert all(torch.equal(a, b) for a, b in zip(e + [db], first))


def test_rows_past_2_31_elements():
    """Rows so far apart that the last ones lie behind 2^31 elements."""
    from paper_2608_02625_gb300 import binding as B
    N, d, f, far = 260, 64, 128, 9_000_000

    def apart(t):
        view = torch.empty(N * far, dtype=BF, device=dev()).as_strided(t.shape, (far, 1))
        view.copy_(t)
        return view

    x, wg, wu = block(N, d, f)
    x = apart(x)
    out = apart(torch.zeros(N, f, dtype=BF, device=dev()))
    B.dlm_gated_linear(x, wg, wu, 1, out, None, None)
    check_gated(x, wg, wu, "silu", out)
    residual = apart(rand(N, f, seed=3))
    B.dlm_linear(x, wg, None, 0, residual, out, residual_pre := apart(out), linear_ws(N, f, d))
    check_linear(x, wg, None, "none", residual, out, residual_pre)
    del residual, residual_pre
    dout = out
    dx = apart(torch.zeros(N, d, dtype=BF, device=dev()))
    dw = torch.empty_like(wg)
    B.dlm_linear_grad(dout, x, wg, None, 0, None, dx, dw, None, linear_grad_ws(N, f, d))
    check_linear_grad(dout, x, wg, None, "none", None, dx, dw, None)
    no_error()


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("N", [3, 200])
def test_gradients_are_differences(N, act):
    """Along random directions: the sum of dout * out changes as the gradients say. The forward
    pass in fp64 by the oracle, so only the gradients' own errors remain (bf16: 2^-7 of their size)."""
    from paper_2608_02625_gb300 import binding as B
    d, f = 64, 136
    x, wg, wu = block(N, d, f)
    dout, gate, up = rand(N, f, seed=1), torch.empty(N, f, dtype=BF, device=dev()), torch.empty(N, f, dtype=BF, device=dev())
    out, dx, dwg, dwu = torch.empty_like(gate), torch.empty_like(x), torch.empty_like(wg), torch.empty_like(wu)
    B.dlm_gated_linear(x, wg, wu, ACTS[act], out, gate, up)
    B.dlm_gated_linear_grad(dout, x, wg, wu, gate, up, ACTS[act], None, dx, dwg, dwu, grad_ws(N, f, d))
    D = host(dout)
    rng = np.random.default_rng(0)
    at = [host(t) for t in (x, wg, wu)]
    for k, g in enumerate((dx, dwg, dwu)):
        way = rng.standard_normal(at[k].shape)
        h = 1e-5
        ends = []
        for sign in (1, -1):
            moved = list(at)
            moved[k] = at[k] + sign * h * way
            ends.append((D * oracle.gated_linear(*moved, act)[0]).sum())
        change, told = (ends[0] - ends[1]) / (2 * h), (host(g) * way).sum()
        size = np.sqrt((host(g) ** 2).sum())  # a direction's share of errors of 2^-7 each is as random as the direction
        assert abs(change - told) <= 6 * 2.0 ** -7 * size
