"""Every form that the feed-forward block's products take, against the oracle in fp64: pairs of CTAs
with tiles of 256 and 128 columns and accumulators that are used again, single CTAs of every width
and split, both gradients in one launch and apart, the bias's gradient in runs; at sizes whose last
tiles and last step of K are ragged (block_forms), and at a training batch's own, by samples.

Inputs lie in buffers of NaN, outputs in canary-filled ones. Tolerances as in block_util, with the
roundings that there are: K is joined from eight CTAs at most, and a bias's gradient adds the rows of
a thread one after another, then the 8 or 32 threads of a column, then up to 8 CTAs and 76 runs."""
import numpy as np
import pytest
import torch

import block_util
import oracle
from block_forms import BIAS, COLS, GATED, GRADIENTS, Plans
from block_util import (ACTS, BF, F32, HALF, STEP, TINY, U32, Guarded, check_gated, check_gated_grad, check_linear, check_linear_grad, dev,
                        host, rand, slope_error, within, workspace)

pytestmark = pytest.mark.gpu

NAMES = list(ACTS)


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    return Plans(str(tmp_path_factory.mktemp("plans")))


@pytest.fixture(autouse=True)
def joined_from_eight(monkeypatch):
    monkeypatch.setattr(block_util, "length", lambda K: (K / 16 + 4) * STEP + 8 * U32)


@pytest.fixture(autouse=True)
def no_error():
    from paper_2608_02625_gb300 import binding as B
    B.device_error(clear=True)
    yield
    assert B.device_error(clear=True) == 0


def inside_nan(t, row=8, offset=8):
    """t in a buffer of NaN: in front, behind the last row and, `row` of them, between rows."""
    rows, cols = t.shape
    buf = torch.full((offset + (rows + 300) * (cols + row),), float("nan"), dtype=t.dtype, device=dev())
    view = buf.as_strided(t.shape, (cols + row, 1), offset)
    view.copy_(t)
    return view


def weights(f, d, seed):
    return inside_nan(rand(f, d, seed=seed, std=d ** -0.5))


def other(gd, given, like, out, seed):
    """(what is passed as add or residual, what it holds)"""
    if given == "no":
        return None, None
    r = rand(*like, seed=seed)
    if given == "itself":
        out.copy_(r)
        return out, r
    r = gd.like(r, row=like[1] + 1, offset=3)
    return r, r


def grad_ws(B, count, N, m, k, gd):
    size = B.dlm_gated_linear_grad_workspace_bytes if count == 2 else B.dlm_linear_grad_workspace_bytes
    return workspace(size, N, m, k, gd=gd)


def name(case):
    return "-".join(map(str, case))


# ---------------------------------------------------------------- values

@pytest.mark.parametrize("case", GATED, ids=name)
def test_gated(plans, case):
    from paper_2608_02625_gb300 import binding as B
    N, d, f, form = case
    assert plans.gated(N, d, f) == form
    i = GATED.index(case)
    x, wg, wu = inside_nan(rand(N, d, seed=i)), weights(f, d, 1), weights(f, d, 2)
    for keep, act in ((True, NAMES[i % 3]), (False, NAMES[(i + 1) % 3])):
        gd = Guarded()
        out = gd.empty(N, f, dtype=BF, row=f + 8)
        gate, up = (gd.empty(N, f, dtype=BF, offset=8), gd.empty(N, f, dtype=BF, row=f + 24)) if keep else (None, None)
        B.dlm_gated_linear(x, wg, wu, ACTS[act], out, gate, up)
        gd.check()
        check_gated(x, wg, wu, act, out, gate, up, where=act)


@pytest.mark.parametrize("wide", [True, False], ids=["aligned", "any"])
@pytest.mark.parametrize("case", COLS, ids=name)
def test_projection(plans, case, wide):
    """wide: rows of 16 bytes' alignment, which are moved so; else none."""
    from paper_2608_02625_gb300 import binding as B
    N, k, m, form = case
    assert plans.cols(N, k, m) == form
    i = COLS.index(case) + wide
    act, bias, given = NAMES[i % 3], (BF, F32, None)[i % 3], ("other", "itself", "no")[(i // 2) % 3]
    x, w = inside_nan(rand(N, k, seed=i)), weights(m, k, 1)
    gd = Guarded()
    more, at = (8, 8) if wide else (5, 3)
    b = None if bias is None else gd.like(rand(m, seed=2, std=0.5, dtype=bias), offset=1)
    out, pre = gd.empty(N, m, dtype=BF, row=m + more, offset=at), gd.empty(N, m, dtype=BF, row=m + 2 * more, offset=at)
    r, held = (gd.like(rand(N, m, seed=3), row=m + 8),) * 2 if wide and given == "other" else other(gd, given, (N, m), out, 3)
    B.dlm_linear(x, w, b, ACTS[act], r, out, pre, None)
    gd.check()
    check_linear(x, w, b, act, held, out, pre)
    # without what may be left out: the same bits where nothing else is added
    plain, again = gd.empty(N, m, dtype=BF, row=m + more, offset=at), gd.empty(N, m, dtype=BF)
    B.dlm_linear(x, w, b, ACTS[act], None, plain, None, None)
    B.dlm_linear(x, w, None, 0, None, again, None, None)
    gd.check()
    check_linear(x, w, b, act, None, plain)
    check_linear(x, w, None, "none", None, again)


@pytest.mark.parametrize("case", GRADIENTS, ids=name)
def test_gradients(plans, case):
    """With everything, then each by itself: dx and dW alone have the bits that they have together."""
    from paper_2608_02625_gb300 import binding as B
    count, N, k, m, *forms = case
    assert plans.gradients(count, N, k, m) == tuple(forms)
    i = GRADIENTS.index(case)
    act, given = NAMES[i % 3], ("other", "itself", "no")[(i // 2) % 3]
    x, dout = inside_nan(rand(N, k, seed=i)), inside_nan(rand(N, m, seed=5))
    w = [weights(m, k, 1 + j) for j in range(count)]
    saved = [inside_nan(rand(N, m, seed=6 + j, std=2.0)) for j in range(2)]
    gd = Guarded()
    dx = gd.empty(N, k, dtype=BF, row=k + (8 if i % 2 else 3), offset=0 if i % 2 else 1)
    dw = [gd.empty(m, k, dtype=BF, row=k + 8 * (j + 1)) for j in range(count)]
    db = gd.empty(m, dtype=(BF, F32)[i % 2], offset=1)
    add, held = other(gd, given, (N, k), dx, 9)
    held = None if held is None else held.clone()
    ws = grad_ws(B, count, N, m, k, gd)

    def call(dx, dw, db, add):
        if count == 2:
            B.dlm_gated_linear_grad(dout, x, *w, *saved, ACTS[act], add, dx, *(dw or (None, None)), ws)
        else:
            B.dlm_linear_grad(dout, x, w[0], saved[0] if act != "none" else None, ACTS[act], add, dx, *(dw or (None,)), db, ws)

    call(dx, dw, db, add)
    gd.check()
    if count == 2:
        check_gated_grad(dout, x, *w, *saved, act, held, dx, *dw)
    else:
        check_linear_grad(dout, x, w[0], saved[0] if act != "none" else None, act, held, dx, dw[0], None)
        check_bias(plans, dout, saved[0], act, db)
    one, several = gd.empty(N, k, dtype=BF), [gd.empty(m, k, dtype=BF) for _ in range(count)]
    call(one, None, None, held)
    call(None, several, None, None)
    gd.check()
    assert torch.equal(one, dx) and all(torch.equal(a, b) for a, b in zip(several, dw))


def check_bias(plans, dout, pre, act, db):
    D, Z = host(dout), host(pre)
    dz = D if act == "none" else D * oracle.activation(act, Z)[1]
    e = 0.0 * dz if act == "none" else np.abs(D) * slope_error(act, Z) + 2 * U32 * np.abs(dz)
    lanes, runs, ranks = plans.bias(*D.shape)
    threads = 256 // lanes
    adds = -(-len(D) // (runs * ranks * threads)) + 1 + threads + ranks + runs
    err = e.sum(0) + adds * U32 * (np.abs(dz) + e).sum(0)
    within(host(db), dz.sum(0), err + HALF[db.dtype] * (np.abs(dz.sum(0)) + err) + TINY, "dbias")


@pytest.mark.parametrize("act", ["none", "gelu"])
@pytest.mark.parametrize("case", BIAS, ids=lambda c: f"{c[0]}-{c[1]}-" + "_".join(map(str, c[2])))
def test_bias_gradients(plans, case, act):
    """Alone, and beside the others: the same bits."""
    from paper_2608_02625_gb300 import binding as B
    N, m, split = case
    assert plans.bias(N, m) == split
    k = 8
    x, w = inside_nan(rand(N, k, seed=1)), weights(m, k, 2)
    dout, pre = inside_nan(rand(N, m, seed=3)), inside_nan(rand(N, m, seed=4, std=2.0))
    gd = Guarded()
    ws = grad_ws(B, 1, N, m, k, gd)
    for dtype in (BF, F32):
        alone, beside = gd.empty(m, dtype=dtype, offset=1), gd.empty(m, dtype=dtype)
        dx, dw = gd.empty(N, k, dtype=BF), gd.empty(m, k, dtype=BF)
        z = None if act == "none" else pre
        B.dlm_linear_grad(dout, x, w, z, ACTS[act], None, None, None, alone, ws)
        B.dlm_linear_grad(dout, x, w, z, ACTS[act], None, dx, dw, beside, ws)
        gd.check()
        check_bias(plans, dout, pre, act, alone)
        assert torch.equal(alone, beside)
    check_linear_grad(dout, x, w, z, act, None, dx, dw, None)


def test_weights_gradients_of_many_tiles(plans):
    """Few rows and many tiles of dW: every CTA writes several, one under the next, in the shared
    launch (one CTA an SM) and by themselves (two)."""
    from paper_2608_02625_gb300 import binding as B
    for N, k, m in ((21, 1032, 4104), (64, 1032, 8200), (100, 2056, 4104)):
        assert plans.gradients(2, N, k, m)[::2] == ("together", "few128/1") and 2 * -(-k // 128) * -(-m // 128) > 3 * 152
        x, dout = inside_nan(rand(N, k, seed=1)), inside_nan(rand(N, m, seed=5))
        w, saved = [weights(m, k, 1 + j) for j in range(2)], [inside_nan(rand(N, m, seed=6 + j, std=2.0)) for j in range(2)]
        gd = Guarded()
        dx, dw, alone = gd.empty(N, k, dtype=BF), [gd.empty(m, k, dtype=BF) for _ in range(2)], [gd.empty(m, k, dtype=BF) for _ in range(2)]
        ws = grad_ws(B, 2, N, m, k, gd)
        B.dlm_gated_linear_grad(dout, x, *w, *saved, 1, None, dx, *dw, ws)
        B.dlm_gated_linear_grad(dout, x, *w, *saved, 1, None, None, *alone, ws)
        gd.check()
        check_gated_grad(dout, x, *w, *saved, "silu", None, dx, *dw)
        assert all(torch.equal(a, b) for a, b in zip(alone, dw))


# ---------------------------------------------------------------- a training batch, by samples

N, D, F = 16384, 2048, 8192
ROWS = sorted({0, 1, 127, 128, 255, 256, 4095, 4096, 9999, N - 257, N - 256, N - 129, N - 128, N - 1, *range(37, N, 397)})
COLUMNS = sorted({0, 1, 63, 64, 127, 128, 255, 256, 2047, F // 2, F - 257, F - 256, F - 1, *range(53, F, 211)})


@pytest.fixture(scope="module")
def batch():
    g = torch.Generator(device=dev()).manual_seed(3)
    r = lambda *s, std=1.0: torch.empty(*s, dtype=BF, device=dev()).normal_(0.0, std, generator=g)  # noqa: E731
    return dict(x=r(N, D), wg=r(F, D, std=D ** -0.5), wu=r(F, D, std=D ** -0.5), wd=r(D, F, std=F ** -0.5), h=r(N, F), gate=r(N, F), up=r(N, F),
                dout=r(N, F), add=r(N, D))


def test_a_batch_gated(plans, batch):
    from paper_2608_02625_gb300 import binding as B
    assert plans.gated(N, D, F) == "pairs256"
    b, e = batch, [torch.empty(N, F, dtype=BF, device=dev()) for _ in range(4)]
    B.dlm_gated_linear(b["x"], b["wg"], b["wu"], 1, *e[:3])
    B.dlm_gated_linear(b["x"], b["wg"], b["wu"], 1, e[3], None, None)
    assert torch.equal(e[0], e[3])
    check_gated(b["x"][ROWS], b["wg"], b["wu"], "silu", *[t[ROWS] for t in e[:3]], where="rows")
    check_gated(b["x"], b["wg"][COLUMNS], b["wu"][COLUMNS], "silu", *[t[:, COLUMNS] for t in e[:3]], where="columns")


def test_a_batch_projected_back(plans, batch):
    from paper_2608_02625_gb300 import binding as B
    assert plans.cols(N, F, D) == "pairs256"
    b, bias = batch, rand(D, seed=8, dtype=F32)
    y, pre = (torch.empty(N, D, dtype=BF, device=dev()) for _ in range(2))
    B.dlm_linear(b["h"], b["wd"], bias, 2, b["add"], y, pre, None)
    check_linear(b["h"][ROWS], b["wd"], bias, "gelu", b["add"][ROWS], y[ROWS], pre[ROWS], where="rows")
    cols = [c for c in COLUMNS if c < D]
    check_linear(b["h"], b["wd"][cols], bias[cols], "gelu", b["add"][:, cols], y[:, cols], pre[:, cols], where="columns")


def test_a_batchs_gated_gradients(plans, batch):
    from paper_2608_02625_gb300 import binding as B
    assert plans.gradients(2, N, D, F) == ("apart", "pairs256", "pairs256")
    b = batch
    dx, dwg, dwu = torch.empty_like(b["x"]), torch.empty_like(b["wg"]), torch.empty_like(b["wu"])
    B.dlm_gated_linear_grad(b["dout"], b["x"], b["wg"], b["wu"], b["gate"], b["up"], 1, b["add"], dx, dwg, dwu,
                            workspace(B.dlm_gated_linear_grad_workspace_bytes, N, F, D))
    some = lambda *names: [b[n][ROWS] for n in names]  # noqa: E731
    d, x, gate, up, add = some("dout", "x", "gate", "up", "add")
    check_gated_grad(d, x, b["wg"], b["wu"], gate, up, "silu", add, dx[ROWS], None, None, where="rows")
    d, gate, up = (b[n][:, COLUMNS] for n in ("dout", "gate", "up"))
    check_gated_grad(d, b["x"], b["wg"][COLUMNS], b["wu"][COLUMNS], gate, up, "silu", None, None, dwg[COLUMNS], dwu[COLUMNS], where="columns")


def test_a_batchs_projection_gradients(plans, batch):
    from paper_2608_02625_gb300 import binding as B
    assert plans.gradients(1, N, D, F) == ("apart", "pairs256", "pairs256") and plans.bias(N, F) == (32, 19, 1)
    b = batch
    dx, dw, db = torch.empty_like(b["x"]), torch.empty_like(b["wg"]), torch.empty(F, device=dev())
    B.dlm_linear_grad(b["dout"], b["x"], b["wg"], b["gate"], 2, b["add"], dx, dw, db, workspace(B.dlm_linear_grad_workspace_bytes, N, F, D))
    check_linear_grad(b["dout"][ROWS], b["x"][ROWS], b["wg"], b["gate"][ROWS], "gelu", b["add"][ROWS], dx[ROWS], None, None, where="rows")
    d, z = b["dout"][:, COLUMNS], b["gate"][:, COLUMNS]
    check_linear_grad(d, b["x"], b["wg"][COLUMNS], z, "gelu", None, None, dw[COLUMNS], None, where="columns")
    full = oracle.activation("gelu", host(z))[1] * host(d)
    err = (np.abs(host(d)) * slope_error("gelu", host(z)) + (2 + N / 152 + 60) * U32 * np.abs(full)).sum(0)
    within(host(db[COLUMNS]), full.sum(0), err * (1 + 2.0 ** -10) + U32 * np.abs(full.sum(0)), "dbias")


# ---------------------------------------------------------------- what else holds for pairs

PAIRS = [(13193, 72, 136), (523, 72, 8680), (2513, 2440, 200), (16227, 328, 552), (2697, 2056, 1064)]


@pytest.mark.parametrize("sizes", PAIRS, ids=str)
def test_the_same_bits_every_time(sizes):
    from paper_2608_02625_gb300 import binding as B
    n, d, f = sizes
    x, wg, wu = rand(n, d, seed=1), rand(f, d, seed=2, std=0.1), rand(f, d, seed=3, std=0.1)
    dout, gate, up, bias = rand(n, f, seed=4), rand(n, f, seed=5), rand(n, f, seed=6), rand(f, seed=7, dtype=F32)
    first = None
    for _ in range(4):
        e = [torch.empty(*s, dtype=BF, device=dev()) for s in ((n, f), (n, f), (n, d), (f, d), (f, d), (n, d), (f, d))]
        db = torch.empty(f, device=dev())
        B.dlm_gated_linear(x, wg, wu, 1, e[0], None, None)
        B.dlm_linear(x, wg, bias, 2, None, e[1], None, None)
        B.dlm_gated_linear_grad(dout, x, wg, wu, gate, up, 1, None, e[2], e[3], e[4], workspace(B.dlm_gated_linear_grad_workspace_bytes, n, f, d))
        B.dlm_linear_grad(dout, x, wg, gate, 2, None, e[5], e[6], db, workspace(B.dlm_linear_grad_workspace_bytes, n, f, d))
        first = first or [t.clone() for t in e + [db]]
        assert all(torch.equal(a, b) for a, b in zip(e + [db], first))


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_bad_rows_stay_alone(plans, bad):
    from paper_2608_02625_gb300 import binding as B
    for n, d, f in ((523, 72, 8680), (13283, 264, 264)):
        at = [4, 261, n - 1]
        assert "pairs" in plans.gated(n, d, f) + plans.cols(n, d, f)
        x, wg, wu = rand(n, d, seed=1), rand(f, d, seed=2, std=0.1), rand(f, d, seed=3, std=0.1)
        x[at, 7] = bad
        out, gate, up, y = (torch.empty(n, f, dtype=BF, device=dev()) for _ in range(4))
        B.dlm_gated_linear(x, wg, wu, 1, out, gate, up)
        B.dlm_linear(x, wg, None, 2, None, y, None, None)
        rest = torch.ones(n, dtype=torch.bool, device=dev())
        rest[at] = False
        for t in (out, gate, up, y):
            assert bool(torch.isfinite(t[rest]).all())
        assert not bool(torch.isfinite(gate[at]).any())
        # a bad row of dout: that row of dx, and all of dW
        dout = rand(n, f, seed=4)
        dout[at, 9] = bad
        dx, dw = torch.empty(n, d, dtype=BF, device=dev()), torch.empty(f, d, dtype=BF, device=dev())
        B.dlm_linear_grad(dout, rand(n, d, seed=5), wg, None, 0, None, dx, dw, None, workspace(B.dlm_linear_grad_workspace_bytes, n, f, d))
        assert bool(torch.isfinite(dx[rest]).all()) and not bool(torch.isfinite(dx[at]).any())
        assert not bool(torch.isfinite(dw[9]).any()) and bool(torch.isfinite(dw[torch.arange(f, device=dev()) != 9]).all())


def test_rows_past_2_31_elements(plans):
    """Rows so far apart that the last ones lie behind 2^31 elements, through pairs of CTAs."""
    from paper_2608_02625_gb300 import binding as B

    def apart(t):
        far = 2 ** 31 // len(t) // 8 * 8 + 4096
        view = torch.empty(len(t) * far, dtype=BF, device=dev()).as_strided(t.shape, (far, 1))
        view.copy_(t)
        return view

    n, d, f = 523, 72, 8680
    assert plans.gated(n, d, f) == "pairs256"
    x, wg, wu = apart(rand(n, d, seed=1)), rand(f, d, seed=2, std=0.1), rand(f, d, seed=3, std=0.1)
    out, gate, up = (apart(torch.zeros(n, f, dtype=BF, device=dev())) for _ in range(3))
    B.dlm_gated_linear(x, wg, wu, 1, out, gate, up)
    check_gated(x, wg, wu, "silu", out, gate, up)
    del out, gate, up, x
    n, k, m = 13283, 264, 264
    assert plans.cols(n, k, m) == "pairs128"
    x, w, residual = apart(rand(n, k, seed=1)), rand(m, k, seed=2, std=0.1), apart(rand(n, m, seed=3))
    out, pre = (apart(torch.zeros(n, m, dtype=BF, device=dev())) for _ in range(2))
    B.dlm_linear(x, w, None, 2, residual, out, pre, None)
    check_linear(x, w, None, "gelu", residual, out, pre)
    del out, pre, residual, x
    n, k, m = 2697, 2056, 1064
    assert plans.gradients(1, n, k, m)[1:] == ("pairs256 few tiles",) * 2
    x, w, dout, pre = apart(rand(n, k, seed=1)), rand(m, k, seed=2, std=0.1), apart(rand(n, m, seed=3)), apart(rand(n, m, seed=4))
    dx, dw, db = apart(torch.zeros(n, k, dtype=BF, device=dev())), torch.empty(m, k, dtype=BF, device=dev()), torch.empty(m, device=dev())
    B.dlm_linear_grad(dout, x, w, pre, 1, dx, dx, dw, db, workspace(B.dlm_linear_grad_workspace_bytes, n, m, k))
    check_linear_grad(dout, x, w, pre, "silu", None, dx, dw, None)
    check_bias(plans, dout, pre, "silu", db)


STEP_SIZES = [(3001, 900, 520, 2568), (2701, 500, 1064, 2056)]


@pytest.mark.parametrize("eight", [False, True], ids=["32bit", "8bit"])
@pytest.mark.parametrize("sizes", STEP_SIZES, ids=str)
def test_results_do_not_depend_on_waiting_between_calls(sizes, eight):
    """A training step whose products are pairs', launch under launch, against one with waits."""
    from test_gpu_block_overlap import run
    waited = run(sizes, True, eight=eight)
    for _ in range(3):
        for a, b in zip(run(sizes, False, eight=eight), waited):
            assert torch.equal(a, b)


def test_step_sizes_take_pairs(plans):
    taken = set()
    for n, _, d, f in STEP_SIZES:
        taken |= {plans.gated(n, d, f), plans.cols(n, f, d), *plans.gradients(2, n, d, f)[1:], *plans.gradients(1, n, f, d)[1:]}
        assert all('pairs' in t for t in (plans.gated(n, d, f), plans.cols(n, f, d), plans.gradients(2, n, d, f)[1]))
    assert {"pairs256", "pairs256 few tiles"} & taken and any("pairs128" in t for t in taken), taken
