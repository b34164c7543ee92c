"""dlm_lmhead_loss and dlm_lmhead_loss_grad against the oracle in fp64.

Tolerances (U = 2^-24, half a step of fp32). A tensor-core product adds 16 terms a step
to an fp32 sum; a step may drop what lies below 2^-22 of the magnitudes added so far, so
a product of length K is off by at most (K / 16 + 4) 2^-22 of its sum of magnitudes.
EX: that bound of the logits, the largest of a row. exp2's argument carries two more
roundings of numbers up to X = max(|x|, |lse|) (in units of log2 e, 1.5), exp2 itself
2^-22; a row's sum has 40 levels of additions, all of positive terms. So lse is off by
at most EX + 8 U X + 2^-21 + 64 U + U |lse|, the loss by EX and a rounding more. In the
gradients, g = dloss (p - hot) is off by |dloss| (p (EX + 8 U X + 2^-21) + 2 U) and rounds
to bf16 (2^-8); the products add their own length's bound, one more rounding for each
piece and split, and round to bf16."""
import numpy as np
import pytest
import torch

import oracle
from train_util import HALF, U32, Guarded, dev, host, within

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
STEP = 2.0 ** -22


def inputs(N, V, d, seed=0, scale=1.0, scored="half"):
    g = torch.Generator(device="cpu").manual_seed(seed + N * 7 + V * 3 + d)
    h = (torch.randn(N, d, generator=g) * scale).to(BF)
    w = (torch.randn(V, d, generator=g) * d ** -0.5).to(BF)
    t = torch.randint(0, V, (N,), generator=g, dtype=torch.int32)
    off = {"all": torch.zeros(N, dtype=torch.bool), "none": torch.ones(N, dtype=torch.bool),
           "half": torch.rand(N, generator=g) < 0.5, "first": torch.arange(N) > 0, "last": torch.arange(N) < N - 1}[scored]
    bad = torch.tensor([-1, V, -100, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32)[torch.arange(N) % 5]
    t = torch.where(off, bad, t)
    h[off] = float("nan")  # never read
    dl = torch.rand(N, generator=g) + 0.25
    dl[off] = float("nan")
    return h.to(dev()), w.to(dev()), t.to(dev()), dl.to(dev())


def bounds(h, w, t):
    """Scored rows, their logits' error bound EX and size X, and the fp64 values."""
    H, W, T = host(h), host(w), t.cpu().numpy()
    rows = oracle.scored_rows(T, len(W))
    H = np.where(np.isin(np.arange(len(T)), rows)[:, None], H, 0.0)
    ex = (H.shape[1] / 16 + 4) * STEP * (np.abs(H) @ np.abs(W).T).max(1)
    x = np.abs(oracle.lm_head_logits(H, W)).max(1)
    return H, W, T, rows, ex, x


def check_loss(h, w, t, loss, lse, where=""):
    H, W, T, rows, ex, x = bounds(h, w, t)
    rl, rs = oracle.lm_head_loss(H, W, T)
    x = np.maximum(x, np.abs(rs))
    b = np.zeros(len(T))
    b[rows] = (ex + 8 * U32 * x + 2.0 ** -21 + 64 * U32)[rows]
    within(host(lse), rs, b + U32 * np.abs(rs), where + " lse")
    within(host(loss), rl, 2 * b + 2 * U32 * (np.abs(rl) + x * (b > 0)), where + " loss")


def check_grad(h, w, t, lse, dl, dh, dw, where="", pieces=1):
    H, W, T, rows, ex, x = bounds(h, w, t)
    S, D = host(lse), np.nan_to_num(host(dl))
    rh, rw, g = oracle.lm_head_loss_grad(H, W, T, S, D)
    x = np.maximum(x, np.abs(S))
    hot = np.zeros_like(g)
    hot[np.arange(len(rows)), T[rows]] = 1.0
    p = np.abs(g + D[rows, None] * hot)  # dloss p
    dg = p * (ex + 8 * U32 * x + 2.0 ** -21)[rows, None] + 2 * U32 * D[rows, None] + 2.0 ** -8 * np.abs(g)
    mags = np.abs(g) + dg
    if dh is not None:
        b = np.zeros_like(rh)
        b[rows] = dg @ np.abs(W) + ((len(W) / 16 + 4) * STEP + (pieces + 64) * U32) * (mags @ np.abs(W))
        within(host(dh), rh, b + HALF[BF] * (np.abs(rh) + b) + 1e-40, where + " d_hidden")
    if dw is not None:
        b = dg.T @ np.abs(H[rows]) + (len(rows) / 16 + 8) * STEP * (mags.T @ np.abs(H[rows]))
        within(host(dw), rw, b + HALF[BF] * (np.abs(rw) + b) + 1e-40, where + " d_weight")


def ws_loss(N, d):
    from paper_2608_02625_gb300 import binding as B
    return torch.full((B.dlm_lmhead_loss_workspace_bytes(N, d),), 0xFF, dtype=torch.uint8, device=dev())


def ws_grad(N, V, d, piece=0):
    from paper_2608_02625_gb300 import binding as B
    return torch.full((B.dlm_lmhead_loss_grad_workspace_bytes(N, V, d, piece),), 0xFF, dtype=torch.uint8, device=dev())


def fp64_lse(h, w, t):
    """What the forward pass leaves, from the oracle (rows not scored: NaN, never read)."""
    H, W, T, rows, _, _ = bounds(h, w, t)
    s = np.full(len(T), np.nan)
    s[rows] = oracle.lm_head_loss(H, W, T)[1][rows]
    return torch.from_numpy(s).float().to(dev())


SIZES = [(1, 1, 8), (3, 7, 8), (1, 300, 64), (128, 256, 64), (130, 1000, 72), (129, 257, 200), (300, 2049, 128), (64, 4099, 512),
         (257, 1024, 320), (5, 151, 2048), (1000, 513, 264), (90, 40000, 64), (520, 1000, 72), (2000, 300, 64), (769, 5000, 128),
         (1025, 2600, 512), (600, 1100, 1024), (513, 300, 2048), (1300, 700, 520), (4200, 600, 264)]


@pytest.mark.parametrize("scored", ["all", "half", "none", "first", "last"])
@pytest.mark.parametrize("N,V,d", SIZES)
def test_loss(N, V, d, scored):
    from paper_2608_02625_gb300 import binding as B
    h, w, t, _ = inputs(N, V, d, scored=scored)
    gd = Guarded()
    loss, lse = gd.empty(N), gd.empty(N)
    B.dlm_lmhead_loss(h, w, t, loss, lse, ws_loss(N, d))
    gd.check()
    assert B.device_error() == 0
    check_loss(h, w, t, loss, lse, f"{N}x{V}x{d} {scored}")


@pytest.mark.parametrize("scored", ["all", "half", "none", "first", "last"])
@pytest.mark.parametrize("N,V,d", SIZES)
def test_gradients(N, V, d, scored):
    from paper_2608_02625_gb300 import binding as B
    h, w, t, dl = inputs(N, V, d, scored=scored)
    lse = fp64_lse(h, w, t)
    gd = Guarded()
    dh, dw = gd.empty(N, d, dtype=BF), gd.empty(V, d, dtype=BF)
    B.dlm_lmhead_loss_grad(h, w, t, lse, dl, dh, dw, ws_grad(N, V, d))
    gd.check()
    assert B.device_error() == 0
    check_grad(h, w, t, lse, dl, dh, dw, f"{N}x{V}x{d} {scored}")


# Products large enough for pairs of CTAs (with half of the rows scored, single ones).
PAIRS = [(700, 11500, 2048), (1300, 12401, 1032), (200, 40001, 2048), (4200, 9301, 264)]


@pytest.mark.parametrize("N,V,d,scored", [(*s, k) for s in PAIRS for k in ("all", "half")] + [(*PAIRS[0], "none"), (*PAIRS[0], "last")])
def test_pairs(N, V, d, scored):
    from paper_2608_02625_gb300 import binding as B
    h, w, t, dl = inputs(N, V, d, seed=13, scored=scored)
    gd = Guarded()
    loss, lse, dh, dw = gd.empty(N), gd.empty(N), gd.empty(N, d, dtype=BF), gd.empty(V, d, dtype=BF)
    B.dlm_lmhead_loss(h, w, t, loss, lse, ws_loss(N, d))
    gd.check()
    check_loss(h, w, t, loss, lse)
    lse = fp64_lse(h, w, t)
    B.dlm_lmhead_loss_grad(h, w, t, lse, dl, dh, dw, ws_grad(N, V, d))
    gd.check()
    assert B.device_error() == 0
    check_grad(h, w, t, lse, dl, dh, dw)


def test_pairs_pieces_and_single_gradients():
    from paper_2608_02625_gb300 import binding as B
    N, V, d, piece = 900, 11300, 1024, 4096
    h, w, t, dl = inputs(N, V, d, seed=14, scored="all")
    t[::50] = -1
    lse = fp64_lse(h, w, t)
    ws = ws_grad(N, V, d, piece)
    dh, dw, dh1, dw1 = (torch.full(s, 7.0, dtype=BF, device=dev()) for s in ((N, d), (V, d), (N, d), (V, d)))
    B.dlm_lmhead_loss_grad(h, w, t, lse, dl, dh, dw, ws)
    B.dlm_lmhead_loss_grad(h, w, t, lse, dl, dh1, None, ws)
    B.dlm_lmhead_loss_grad(h, w, t, lse, dl, None, dw1, ws)
    torch.cuda.synchronize()
    check_grad(h, w, t, lse, dl, dh, dw, "both", 3)
    check_grad(h, w, t, lse, dl, dh1, None, "d_hidden alone", 3)
    assert torch.equal(dw, dw1) and B.device_error() == 0


@pytest.mark.parametrize("offset,gap,wgap", [(1, 0, 0), (3, 7, 16), (8, 16, 8)])
def test_pairs_strides_and_alignment(offset, gap, wgap):
    from paper_2608_02625_gb300 import binding as B
    L, V, d = 130, 20500, 1024
    N, row, wrow = 6 * L, d + gap, d + wgap
    h, w, t, dl = inputs(N, V, d, seed=15, scored="all")
    t[5::90] = V
    gd = Guarded()
    hs, ws_, ts = gd.like(h.view(6, L, d), offset=offset, row=row), gd.like(w, row=wrow), t.view(6, L)
    loss, lse = gd.empty(6, L), gd.empty(6, L)
    B.dlm_lmhead_loss(hs, ws_, ts, loss, lse, ws_loss(N, d))
    gd.check()
    check_loss(h, w, t, loss.view(-1), lse.view(-1))
    dh, dw = gd.empty(6, L, d, dtype=BF, offset=offset, row=row), gd.empty(V, d, dtype=BF, row=wrow)
    B.dlm_lmhead_loss_grad(hs, ws_, ts, lse, dl.view(6, L), dh, dw, ws_grad(N, V, d))
    gd.check()
    check_grad(h, w, t, lse.view(-1), dl, dh.reshape(N, d), dw)


def test_pairs_replayed_with_more_and_fewer_scored_rows():
    """One captured pass over numbers of scored rows that take single CTAs and pairs; the
    same number gives the same bits as without the graph."""
    from paper_2608_02625_gb300 import binding as B
    N, V, d = 900, 9000, 2048
    h, w, all_t, dl = inputs(N, V, d, seed=16, scored="all")
    t = all_t.clone()
    new = lambda: [torch.empty(N, device=dev()), torch.empty(N, device=dev()), torch.empty_like(h), torch.empty_like(w)]  # noqa: E731
    a, b, first, out = ws_loss(N, d), ws_grad(N, V, d), new(), new()

    def go(o):
        B.dlm_lmhead_loss(h, w, t, o[0], o[1], a)
        B.dlm_lmhead_loss_grad(h, w, t, o[1], dl, o[2], o[3], b)

    go(first)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        go(out)
    for n in (100, N, 600, 0, N):
        t.copy_(torch.where(torch.arange(N, device=dev()) % N < n, all_t, -1))
        graph.replay()
        torch.cuda.synchronize()
        check_loss(h, w, t, out[0], out[1], f"{n} of {N}")
        check_grad(h, w, t, out[1], dl, out[2], out[3], f"{n} of {N}")
    assert B.device_error() == 0
    for x, y in zip(first, out):
        assert torch.equal(x, y)


@pytest.mark.parametrize("weights", ["equal", "any"])
@pytest.mark.parametrize("N,V,d,piece", [(200, 3001, 128, 0), (200, 3001, 128, 1024), (600, 2500, 512, 0), (1, 300, 64, 0),
                                         (800, 13000, 1024, 0)])
def test_the_targets_terms_keep_their_precision(N, V, d, piece, weights):
    """The bounds of check_grad but for the target's term, which is most of a row's
    gradient. In d_hidden it is not rounded to bf16: two fp32 roundings instead of 2^-8.
    With equal weights it is rounded as 2^k (1 - p) in d_weight, between 1/2 and 1 a number
    of steps of 2^-8, 1 one of them: off by at most min(p, 2^-9). The equal weight is one
    that bf16 misses by 0.9 of half a step."""
    from paper_2608_02625_gb300 import binding as B
    h, w, t, dl = inputs(N, V, d, seed=7, scored="all")
    if weights == "equal":
        dl.fill_(2.0 ** -6 * (1 + 0.9 * 2.0 ** -8))
    lse = fp64_lse(h, w, t)
    dh, dw = torch.empty_like(h), torch.empty_like(w)
    B.dlm_lmhead_loss_grad(h, w, t, lse, dl, dh, dw, ws_grad(N, V, d, piece))
    H, W, T, rows, ex, x = bounds(h, w, t)
    S, D = host(lse), host(dl)
    rh, rw, g = oracle.lm_head_loss_grad(H, W, T, S, D)
    x = np.maximum(x, np.abs(S))
    at = np.arange(N), T
    hot = np.zeros_like(g)
    hot[at] = 1.0
    p = np.abs(g + D[:, None] * hot)
    dg = p * (ex + 8 * U32 * x + 2.0 ** -21)[:, None] + 4 * U32 * D[:, None]
    mags = np.abs(g) * (1 + 2.0 ** -8) + dg
    off = 2.0 ** -8 * np.abs(g)
    off[at] = 2 * U32 * np.abs(g[at])
    b = (dg + off) @ np.abs(W) + ((V / 16 + 4) * STEP + 80 * U32) * (mags @ np.abs(W))
    within(host(dh), rh, b + HALF[BF] * (np.abs(rh) + b) + 1e-40, "d_hidden")
    if weights == "equal":
        off[at] = np.minimum(p[at], 2.0 ** -9 * D) + 2 * U32 * np.abs(g[at])
        b = (dg + off).T @ np.abs(H) + (N / 16 + 8) * STEP * (mags.T @ np.abs(H))
        within(host(dw), rw, b + HALF[BF] * (np.abs(rw) + b) + 1e-40, "d_weight")
    assert B.device_error() == 0


@pytest.mark.parametrize("N,V,d", [(900, 1500, 1024), (300, 700, 1024), (4200, 300, 256)])
def test_replayed_with_more_and_fewer_scored_rows(N, V, d):
    """One captured pass over numbers of scored rows that take single CTAs and pairs."""
    from paper_2608_02625_gb300 import binding as B
    h, w, all_t, dl = inputs(N, V, d, seed=12, scored="all")
    t = all_t.clone()
    loss, lse, dh, dw = torch.empty(N, device=dev()), torch.empty(N, device=dev()), torch.empty_like(h), torch.empty_like(w)
    a, b = ws_loss(N, d), ws_grad(N, V, d, 512)

    def go():
        B.dlm_lmhead_loss(h, w, t, loss, lse, a)
        B.dlm_lmhead_loss_grad(h, w, t, lse, dl, dh, dw, b)

    go()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        go()
    order = torch.randperm(N, generator=torch.Generator().manual_seed(1))
    for n in (N, 384, 385, 128, 129, 256, 257, 0, 1, N - 1):
        if n > N:
            continue
        keep = torch.zeros(N, dtype=torch.bool)
        keep[order[:n]] = True
        t.copy_(torch.where(keep.to(dev()), all_t, -1))
        graph.replay()
        torch.cuda.synchronize()
        check_loss(h, w, t, loss, lse, f"{n} of {N}")
        check_grad(h, w, t, lse, dl, dh, dw, f"{n} of {N}", -(-V // 512))
    assert B.device_error() == 0


@pytest.mark.parametrize("N,V", [(128, 300), (100, 1), (77, 5)])
def test_many_rows_of_one_token(N, V):
    from paper_2608_02625_gb300 import binding as B
    d = 128
    h, w, t, dl = inputs(N, V, d, seed=10, scored="all")
    t.fill_(V - 1)
    lse = fp64_lse(h, w, t)
    dh, dw = torch.empty_like(h), torch.empty_like(w)
    B.dlm_lmhead_loss_grad(h, w, t, lse, dl, dh, dw, ws_grad(N, V, d))
    assert B.device_error() == 0
    check_grad(h, w, t, lse, dl, dh, dw)


@pytest.mark.parametrize("bad", [0.0, float("inf"), float("nan"), -0.75, 1e-39])
def test_any_weight_of_the_first_row(bad):
    """Whatever the first scored row's weight is, the other rows' gradients are theirs."""
    from paper_2608_02625_gb300 import binding as B
    N, V, d = 60, 500, 64
    h, w, t, dl = inputs(N, V, d, seed=8, scored="all")
    lse = fp64_lse(h, w, t)
    dl[0] = bad
    dh, dw = torch.empty_like(h), torch.empty_like(w)
    B.dlm_lmhead_loss_grad(h, w, t, lse, dl, dh, dw, ws_grad(N, V, d))
    if np.isfinite(bad):
        check_grad(h, w, t, lse, dl.abs(), dh * torch.where(dl < 0, -1, 1)[:, None].to(BF), None)
        keep = dl.clone()
        keep[0] = 0.0
        dh1, dw1 = torch.empty_like(h), torch.empty_like(w)
        B.dlm_lmhead_loss_grad(h, w, t, lse, keep, dh1, dw1, ws_grad(N, V, d))
        if bad in (0.0, 1e-39):
            assert torch.equal(dw, dw1)
    else:
        assert not bool(torch.isfinite(dh[0]).any())
        keep = t.clone()
        keep[0] = -1
        check_grad(h, w, keep, lse, dl, torch.cat([torch.zeros_like(dh[:1]), dh[1:]]), None)


@pytest.mark.parametrize("scored", ["half", "last"])
def test_more_rows_than_the_gathering_ctas_take_at_once(scored):
    from paper_2608_02625_gb300 import binding as B
    N, V, d = 270_003, 40, 16
    h, w, t, dl = inputs(N, V, d, seed=6, scored=scored)
    gd = Guarded()
    loss, lse, dh, dw = gd.empty(N), gd.empty(N), gd.empty(N, d, dtype=BF), gd.empty(V, d, dtype=BF)
    B.dlm_lmhead_loss(h, w, t, loss, lse, ws_loss(N, d))
    gd.check()
    check_loss(h, w, t, loss, lse)
    lse = fp64_lse(h, w, t)
    B.dlm_lmhead_loss_grad(h, w, t, lse, dl, dh, dw, ws_grad(N, V, d))
    gd.check()
    assert B.device_error() == 0
    check_grad(h, w, t, lse, dl, dh, dw)


@pytest.mark.parametrize("N,V,d,piece", [(300, 2049, 128, 256), (300, 2049, 128, 1024), (64, 4099, 512, 1024), (20, 1300, 72, 512),
                                         (700, 900, 64, 256), (1500, 3000, 320, 1024), (700, 2000, 512, 512)])
def test_pieces_and_single_gradients(N, V, d, piece):
    """Several pieces of the vocabulary; d_hidden or d_weight alone (the sums of d_hidden
    may then be split otherwise)."""
    from paper_2608_02625_gb300 import binding as B
    h, w, t, dl = inputs(N, V, d, seed=1)
    lse = fp64_lse(h, w, t)
    ws = ws_grad(N, V, d, piece)
    dh, dw, dh1, dw1 = (torch.full(s, 7.0, dtype=BF, device=dev()) for s in ((N, d), (V, d), (N, d), (V, d)))
    B.dlm_lmhead_loss_grad(h, w, t, lse, dl, dh, dw, ws)
    B.dlm_lmhead_loss_grad(h, w, t, lse, dl, dh1, None, ws)
    B.dlm_lmhead_loss_grad(h, w, t, lse, dl, None, dw1, ws)
    torch.cuda.synchronize()
    check_grad(h, w, t, lse, dl, dh, dw, f"pieces of {piece}", -(-V // piece))
    check_grad(h, w, t, lse, dl, dh1, None, f"d_hidden alone, pieces of {piece}", -(-V // piece))
    assert torch.equal(dw, dw1) and B.device_error() == 0


@pytest.mark.parametrize("L,d", [(35, 64), (100, 512)], ids=["single_ctas", "pairs"])
@pytest.mark.parametrize("offset,gap,wgap", [(0, 8, 8), (1, 0, 0), (3, 7, 16), (8, 16, 0)])
def test_strides_and_alignment(offset, gap, wgap, L, d):
    from paper_2608_02625_gb300 import binding as B
    N, V, row, wrow = 6 * L, 700, d + gap, d + wgap
    h, w, t, dl = inputs(N, V, d, seed=2)
    gd = Guarded()
    hs, ws_, ts = gd.like(h.view(6, L, d), offset=offset, row=row), gd.like(w, row=wrow), t.view(6, L)
    loss, lse = gd.empty(6, L), gd.empty(6, L)
    B.dlm_lmhead_loss(hs, ws_, ts, loss, lse, ws_loss(N, d))
    gd.check()
    check_loss(h, w, t, loss.view(-1), lse.view(-1))
    dh, dw = gd.empty(6, L, d, dtype=BF, offset=offset, row=row), gd.empty(V, d, dtype=BF, row=wrow)
    B.dlm_lmhead_loss_grad(hs, ws_, ts, lse, dl.view(6, L), dh, dw, ws_grad(N, V, d))
    gd.check()
    check_grad(h, w, t, lse.view(-1), dl, dh.reshape(N, d), dw)


@pytest.mark.parametrize("scale", [30.0, 300.0])
def test_peaked_rows(scale):
    """Logits far apart: most probabilities underflow, targets among the unlikely ones."""
    from paper_2608_02625_gb300 import binding as B
    N, V, d = 150, 3000, 128
    h, w, t, dl = inputs(N, V, d, scale=scale, scored="all")
    t[::3] = torch.from_numpy((host(h) @ host(w).T).argmax(1)[::3]).int().to(dev())
    loss, lse = torch.empty(N, device=dev()), torch.empty(N, device=dev())
    B.dlm_lmhead_loss(h, w, t, loss, lse, ws_loss(N, d))
    check_loss(h, w, t, loss, lse)
    dh, dw = torch.empty_like(h), torch.empty_like(w)
    B.dlm_lmhead_loss_grad(h, w, t, lse, dl, dh, dw, ws_grad(N, V, d))
    check_grad(h, w, t, lse, dl, dh, dw)


def test_not_finite_rows_stay_alone():
    from paper_2608_02625_gb300 import binding as B
    N, V, d = 140, 500, 64
    h, w, t, _ = inputs(N, V, d, scored="all")
    out = [torch.empty(N, device=dev()) for _ in range(4)]
    B.dlm_lmhead_loss(h, w, t, out[0], out[1], ws_loss(N, d))
    h[7, 3], h[131, 5] = float("nan"), float("inf")
    B.dlm_lmhead_loss(h, w, t, out[2], out[3], ws_loss(N, d))
    bad = torch.zeros(N, dtype=torch.bool, device=dev())
    bad[7] = bad[131] = True
    for a, b in ((out[0], out[2]), (out[1], out[3])):
        assert bool(torch.isnan(b[bad]).all()) and torch.equal(a[~bad], b[~bad])
    # a weight row of NaN reaches every row, wherever it lies in a tile
    h, w, t, _ = inputs(N, V, d, scored="all")
    for lo, hi in ((0, 32), (255, 256), (499, 500), (0, 500)):
        bad_w = w.clone()
        bad_w[lo:hi] = float("nan")
        B.dlm_lmhead_loss(h, bad_w, t, out[2], out[3], ws_loss(N, d))
        assert bool(torch.isnan(out[2]).all()) and bool(torch.isnan(out[3]).all())
    assert B.device_error() == 0


def test_no_rows():
    from paper_2608_02625_gb300 import binding as B
    w = torch.randn(30, 64).to(BF).to(dev())
    h, t, f = torch.empty(0, 64, dtype=BF, device=dev()), torch.empty(0, dtype=torch.int32, device=dev()), torch.empty(0, device=dev())
    ws = torch.empty(16, dtype=torch.uint8, device=dev())
    B.dlm_lmhead_loss(h, w, t, f, f.clone(), ws)
    gd = Guarded()
    dw = gd.empty(30, 64, dtype=BF, row=72)
    B.dlm_lmhead_loss_grad(h, w, t, f, f.clone(), torch.empty_like(h), dw, ws)
    gd.check()
    assert bool((dw == 0).all())


def test_against_the_fused_reduction():
    """The scored rows' lse equals that of dlm_lmhead_confidence, and a row's loss is -ln
    of its confidence where the target is the argmax, within both calls' tolerances."""
    from paper_2608_02625_gb300 import binding as B
    N, V, d = 200, 5000, 256
    h, w, t, _ = inputs(N, V, d, seed=4, scale=2.0, scored="all")
    am, cf, ls = torch.empty(N, dtype=torch.int32, device=dev()), torch.empty(N, device=dev()), torch.empty(N, device=dev())
    B.dlm_lmhead_confidence(h, w, am, cf, ls, torch.empty(B.dlm_lmhead_workspace_bytes(N), dtype=torch.uint8, device=dev()))
    loss, lse = torch.empty(N, device=dev()), torch.empty(N, device=dev())
    B.dlm_lmhead_loss(h, w, am, loss, lse, ws_loss(N, d))
    check_loss(h, w, am, loss, lse)
    assert float((lse - ls).abs().max()) <= 4e-5 * float(ls.abs().max())
    assert float((torch.exp(-loss) / cf - 1).abs().max()) <= 1e-4


def test_gradients_against_differences():
    """d_hidden against differences of the GPU's own loss: steps that bf16 holds exactly."""
    from paper_2608_02625_gb300 import binding as B
    N, V, d, step = 4, 37, 16, 2.0 ** -5
    g = torch.Generator(device="cpu").manual_seed(11)
    h = (torch.randint(-64, 65, (N, d), generator=g).float() / 64).to(BF).to(dev())
    w = (torch.randn(V, d, generator=g) * 0.5).to(BF).to(dev())
    t = torch.tensor([3, -1, 36, 0], dtype=torch.int32, device=dev())
    dl = torch.tensor([1.0, 1.0, 0.5, 2.0], device=dev())
    loss, lse, ws = torch.empty(N, device=dev()), torch.empty(N, device=dev()), ws_loss(N, d)

    def value(h):
        B.dlm_lmhead_loss(h, w, t, loss, lse, ws)
        return float((loss.double() * dl.double()).sum())

    value(h)
    dh, dw = torch.empty_like(h), torch.empty_like(w)
    B.dlm_lmhead_loss_grad(h, w, t, lse.clone(), dl, dh, dw, ws_grad(N, V, d))
    for r in range(N):
        for k in range(d):
            up, down = h.clone(), h.clone()
            up[r, k] += step
            down[r, k] -= step
            if float(up[r, k]) - float(down[r, k]) != 2 * step:
                continue  # bf16 does not hold both
            diff = (value(up) - value(down)) / (2 * step)
            # third derivative of lse along one weight column: at most 6 max|w|^3
            curve = step ** 2 * float(w[:, k].abs().max()) ** 3 * 2.0
            assert abs(diff - float(dh[r, k])) <= 2.0 ** -7 * abs(diff) + curve + 2.0 ** -8 * 0.1 + 1e-4


@pytest.mark.parametrize("N,V,d", [(500, 3001, 192), (700, 3001, 1024)])
def test_same_bits_again_on_another_stream_and_replayed(N, V, d):
    from paper_2608_02625_gb300 import binding as B
    h, w, t, dl = inputs(N, V, d, seed=5)
    new = lambda: [torch.empty(N, device=dev()), torch.empty(N, device=dev()), torch.empty_like(h), torch.empty_like(w)]  # noqa: E731

    def go(o, a, b):
        B.dlm_lmhead_loss(h, w, t, o[0], o[1], a)
        B.dlm_lmhead_loss_grad(h, w, t, o[1], dl, o[2], o[3], b)

    first, second, third = new(), new(), new()
    a, b = ws_loss(N, d), ws_grad(N, V, d, 1024)
    go(first, a, b)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    a2, b2 = ws_loss(N, d), ws_grad(N, V, d, 1024)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        go(second, a2, b2)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        go(third, a, b)
    graph.replay()
    # other targets, fewer scored rows: the same graph follows what is in memory
    t2 = t.clone()
    t2[::2] = -1
    keep = t.clone()
    t.copy_(t2)
    graph.replay()
    check_loss(h, w, t, third[0], third[1])
    check_grad(h, w, t, third[1], dl, third[2], third[3], pieces=3)
    t.copy_(keep)
    graph.replay()
    torch.cuda.synchronize()
    assert B.device_error() == 0
    for x, y, z in zip(first, second, third):
        assert torch.equal(x, y) and torch.equal(x, z)


def test_offsets_past_32_bits():
    """A weight and its gradient of more than 2^31 elements, and hidden states of more than
    2^31, few of them scored; values against fp64 on the GPU."""
    from paper_2608_02625_gb300 import binding as B
    d = 2048
    for N, V, at in ((3, 1_100_000, [5, 600_000, 1_099_999]), (1_100_000, 300, [7, 0, 299])):
        g = torch.Generator(device=dev()).manual_seed(3)
        h = torch.empty(N, d, dtype=BF, device=dev()).normal_(generator=g)
        w = torch.empty(V, d, dtype=BF, device=dev()).normal_(0.0, d ** -0.5, generator=g)
        t = torch.full((N,), -1, dtype=torch.int32, device=dev())
        rows = torch.tensor([0, N // 2, N - 1], device=dev())
        t[rows] = torch.tensor(at, dtype=torch.int32, device=dev())
        loss, lse, dl = torch.empty(N, device=dev()), torch.empty(N, device=dev()), torch.ones(N, device=dev())
        B.dlm_lmhead_loss(h, w, t, loss, lse, torch.empty(B.dlm_lmhead_loss_workspace_bytes(N, d), dtype=torch.uint8, device=dev()))
        x = torch.cat([h[rows].double() @ c.double().T for c in w.split(100_000)], 1)
        ref = torch.logsumexp(x, 1) - x[torch.arange(3), t[rows].long()]
        assert float((loss[rows] - ref).abs().max()) <= 1e-3
        dh, dw = torch.empty_like(h), torch.empty_like(w)
        B.dlm_lmhead_loss_grad(h, w, t, lse, dl, dh, dw,
                               torch.empty(B.dlm_lmhead_loss_grad_workspace_bytes(N, V, d, 65536), dtype=torch.uint8, device=dev()))
        p = torch.exp(x - lse[rows].double()[:, None])
        p[torch.arange(3), t[rows].long()] -= 1.0
        want = sum(p[:, i:i + 100_000] @ w[i:i + 100_000].double() for i in range(0, V, 100_000))
        assert float((dh[rows].double() - want).norm() / want.norm()) <= 2.0 ** -8
        assert int((dh != 0).any(1).sum()) == 3
        for v in (0, at[1], V - 1, V // 2):
            want = p[:, v] @ h[rows].double()
            assert float((dw[v].double() - want).norm()) <= 2.0 ** -7 * float((p[:, v].abs() @ h[rows].double().abs()).norm())
        assert B.device_error() == 0


def test_a_training_step_of_the_last_layer():
    """Norm, loss, both gradients and clipping one after another, as a training program
    calls them, against fp64 autograd of the same step. Between them the norm's output, g,
    d_hidden, d_weight and the clipped gradients round to bf16, each by at most 2^-8
    relative to its values; a logit moves by at most 2^-8 sum |h w| / sqrt(d) in the mean,
    0.01 here, and with it g by 1 %: together below 2^-5 of the result's norm."""
    from paper_2608_02625_gb300 import binding as B
    N, V, d = 600, 2500, 256
    g = torch.Generator(device="cpu").manual_seed(21)
    x = (torch.randn(N, d, generator=g) * 2 + 0.3).to(BF).to(dev())
    nw, nb = (1 + 0.2 * torch.randn(d, generator=g)).to(dev()), (0.2 * torch.randn(d, generator=g)).to(dev())
    w = (torch.randn(V, d, generator=g) * d ** -0.5).to(BF).to(dev())
    t = torch.where(torch.rand(N, generator=g) < 0.3, torch.randint(0, V, (N,), generator=g), V).int().to(dev())
    n = int((t < V).sum())
    dl = torch.full((N,), 1.0 / n, device=dev())

    h, mean, rstd = torch.empty_like(x), torch.empty(N, device=dev()), torch.empty(N, device=dev())
    loss, lse = torch.empty(N, device=dev()), torch.empty(N, device=dev())
    dh, dw, dx, dnw, dnb = (torch.empty_like(s) for s in (x, w, x, nw, nb))
    norm = torch.empty(1, device=dev())
    B.dlm_layer_norm(x, nw, nb, 1e-5, h, mean, rstd)
    B.dlm_lmhead_loss(h, w, t, loss, lse, ws_loss(N, d))
    B.dlm_lmhead_loss_grad(h, w, t, lse, dl, dh, dw, ws_grad(N, V, d, 1024))
    B.dlm_layer_norm_grad(dh, x, nw, mean, rstd, dx, dnw, dnb,
                          torch.empty(B.dlm_layer_norm_grad_workspace_bytes(N, d), dtype=torch.uint8, device=dev()))
    grads = [dw, dnw, dnb]
    B.dlm_clip_grad_norm(grads, grads, 0.05, norm,
                         torch.empty(B.dlm_clip_grad_norm_workspace_bytes(), dtype=torch.uint8, device=dev()))
    torch.cuda.synchronize()
    assert B.device_error() == 0

    X, NW, NB, W = (v.double().cpu().requires_grad_(True) for v in (x, nw, nb, w))
    H = torch.nn.functional.layer_norm(X, (d,), NW, NB, 1e-5)
    ref = torch.nn.functional.cross_entropy(H @ W.T, torch.where(t < V, t, -100).long().cpu(), reduction="mean")
    ref.backward()
    ref = ref.detach()
    total = torch.sqrt(sum((p.grad ** 2).sum() for p in (W, NW, NB)))
    scale = min(1.0, 0.05 / (float(total) + 1e-6))
    assert abs(float(loss.sum() / n) - float(ref)) <= 2.0 ** -7 * float(ref)
    assert abs(float(norm) / float(total) - 1) <= 2.0 ** -5
    for got, want, s in ((dx, X.grad, 1.0), (dw, W.grad, scale), (dnw, NW.grad, scale), (dnb, NB.grad, scale)):
        assert float((got.double().cpu() - s * want).norm() / (s * want).norm()) <= 2.0 ** -5


def test_a_refused_weight_leaves_the_outputs_alone():
    """Rows of the weight 2^40 bytes apart (never read): nothing runs, not even for the rows
    that are not scored."""
    import ctypes

    from paper_2608_02625_gb300 import binding as B
    N, d = 40, 64
    buf = torch.zeros(1 << 20, dtype=torch.uint8, device=dev())  # the weight behind the others
    cut = lambda at, dtype, *s: buf[at:].view(dtype)[:int(np.prod(s))].view(*s)  # noqa: E731
    h, loss, lse = cut(0, BF, N, d), cut(1 << 17, torch.float32, N), cut(2 << 17, torch.float32, N)
    t, dh, dw = cut(3 << 17, torch.int32, N).fill_(-1), cut(4 << 17, BF, N, d), cut(5 << 17, BF, 2, d)
    w = B.describe(cut(7 << 17, BF, 2, d))
    w.stride[0] = 2 ** 39
    for o in (loss, lse, dh, dw):
        o.fill_(7.0)
    dl = torch.ones(N, device=dev())
    ws, wsg = ws_loss(N, d), ws_grad(N, 2, d)
    refs = lambda *ts: [ctypes.byref(B.describe(x) if isinstance(x, torch.Tensor) else x) for x in ts]  # noqa: E731
    torch.cuda.synchronize()
    B._prepare(h, loss)
    assert B.lib.dlm_lmhead_loss(*refs(h, w, t, loss, lse), *B._workspace(ws)) == -4
    assert B.lib.dlm_lmhead_loss_grad(*refs(h, w, t, lse, dl, dh, dw), *B._workspace(wsg)) == -4
    torch.cuda.synchronize()
    for o in (loss, lse, dh, dw):
        assert bool((o == 7.0).all())
