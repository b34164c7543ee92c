"""dlm_adamw against the oracle in fp64.

Tolerances, in roundings of fp32 (U = 2^-24). A coefficient and the clipping factor are
rounded once each, so with M = |beta1 m| + |(1 - beta1) g| the new m is off by at most 6 U M
(two coefficients, two products, the factor, the sum) and the new v, all of whose terms are
positive, by 8 U v; sqrt(v) then by 6 U (half of that, and an approximation good to 2 U). The step's size, lr / (1 - beta1^t) m / (sqrt(v) /
sqrt(1 - beta2^t) + eps): the two corrections by 5 U each (the rounded t ln beta, expm1f of one
ulp, a division or a square root and its reciprocal), the quotient by another 5 (its
approximation is good to 2 ulp); so by 32 U lr / (1 - beta1^t) M / (sqrt(v / (1 - beta2^t)) +
eps) at most. The weight: that, and 3 U |p|, and half a step of its type.
Codes: half a step of e4m3, 2^-4 |x| or 2^-10 of the scale, of a value off by the above and a
scale off by another 2 U; a sqrt(v) above 0 may be held as the smallest code, 2^-9 of the
scale. 8 U on top of each covers them. Squares and codes below fp32's normal range are not among
these inputs, but for those of test_small_second_moments."""
import numpy as np
import pytest
import torch

import oracle
from train_util import HALF, U32, Guarded, dev, host, within

pytestmark = pytest.mark.gpu

BF, F32, U8 = torch.bfloat16, torch.float32, torch.uint8
HYPER = dict(beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1)


class Case:
    """Tensors of one call, in canary-filled buffers, and what they held."""

    def __init__(self, sizes, kind="f32", grads=F32, eight=False, seed=0, offset=0, t=3, lr=1e-2, norm=None, max_norm=np.inf,
                 zeros=False, **hyper):
        from paper_2608_02625_gb300 import binding as B
        g = torch.Generator(device="cpu").manual_seed(seed)
        self.gd, self.kind, self.eight = Guarded(), kind, eight
        self.hyper = {**HYPER, **hyper}
        rnd = lambda n, s: torch.randn(n, generator=g) * s  # noqa: E731
        put = lambda x, dt: self.gd.like(x.to(dev()).to(dt), offset=offset)  # noqa: E731
        p = [rnd(n, 0.02) for n in sizes]
        self.masters = [put(x, F32) for x in p] if kind == "master" else None
        self.params = [put(x, F32 if kind == "f32" else BF) for x in p]
        self.grads = [put(rnd(n, 1e-3), grads if isinstance(grads, torch.dtype) else grads[i % len(grads)])
                      for i, n in enumerate(sizes)]
        m = [torch.zeros(n) if zeros else rnd(n, 3e-4) for n in sizes]
        r = [torch.zeros(n) if zeros else rnd(n, 1e-3).abs() + 1e-5 for n in sizes]
        if eight:
            self.m, self.ms = map(list, zip(*[self.codes(x, put) for x in m]))
            self.v, self.vs = map(list, zip(*[self.codes(x, put) for x in r]))
        else:
            self.m, self.v, self.ms, self.vs = [put(x, F32) for x in m], [put(x * x, F32) for x in r], None, None
        self.lr = torch.full((1,), lr, device=dev())
        self.step = torch.full((1,), t, dtype=torch.int32, device=dev())
        self.norm = None if norm is None else torch.full((1,), norm, device=dev())
        self.max_norm = max_norm
        self.call_hyper = B.AdamwParams(lr=self.lr, step=self.step, norm=self.norm, max_norm=max_norm, **self.hyper)
        self.keep()

    @staticmethod
    def codes(x, put):
        s = torch.from_numpy(oracle.block_scales(x.numpy())).float()
        each = s.repeat_interleave(256)[:x.numel()]
        q = torch.where(each > 0, x / each, torch.zeros_like(x)).clamp(-448, 448).to(torch.float8_e4m3fn).view(U8)
        return put(q, U8), put(s, F32)

    def states(self):
        """m and the second moment as fp64."""
        if self.eight:
            return [[oracle.held(q.cpu().numpy(), z.cpu().numpy()) ** k for q, z in zip(c, s)]
                    for c, s, k in ((self.m, self.ms, 1), (self.v, self.vs, 2))]
        return [[host(x) for x in self.m], [host(x) for x in self.v]]

    def keep(self):
        """What the tensors hold now is what the next check starts from."""
        self.before = [host(x) for x in (self.masters or self.params)], *self.states()

    def run(self):
        from paper_2608_02625_gb300 import binding as B
        B.dlm_adamw(self.params, self.masters, self.grads, self.m, self.v, self.ms, self.vs, self.call_hyper)

    def check(self, t=None, lr=None, where=""):
        self.gd.check()
        h, lr = self.hyper, float(self.lr) if lr is None else lr
        t = max(1, int(self.step)) if t is None else t
        norm = None if self.norm is None else float(self.norm)
        scale = 1.0 if norm is None else min(1.0, self.max_norm / (norm + 1e-6))
        for i, g in enumerate(self.grads):
            p0, m0, v0 = (x[i] for x in self.before)
            g = host(g)
            p, m, v = oracle.adamw(p0, g, m0, v0, t, lr, norm=norm, max_norm=self.max_norm, **h)
            M = np.abs(h["beta1"] * m0) + np.abs((1 - h["beta1"]) * scale * g)
            per = lr / (1 - h["beta1"] ** t) / (np.sqrt(v / (1 - h["beta2"] ** t)) + h["eps"])
            bound = 32 * U32 * per * M + 3 * U32 * (np.abs(p0) + np.abs(p))
            w = f"{where} tensor {i}"
            if self.masters:
                within(host(self.masters[i]), p, bound, w + " master")
                assert torch.equal(self.params[i], self.masters[i].to(BF)), w + " copy"
            else:
                within(host(self.params[i]), p, bound + HALF[self.params[i].dtype] * (np.abs(p) + bound), w + " weight")
            if not self.eight:
                within(host(self.m[i]), m, 6 * U32 * M, w + " m")
                within(host(self.v[i]), v, 8 * U32 * v, w + " v")
                continue
            for codes, scales, x, err, least in ((self.m, self.ms, m, 6 * U32 * M, 2.0 ** -10),
                                                 (self.v, self.vs, np.sqrt(v), 6 * U32 * np.sqrt(v), 2.0 ** -9)):
                s = oracle.block_scales(x)
                top = np.maximum.reduceat(err, np.arange(0, len(err), 256)) if len(err) else err
                within(host(scales[i]), s, (top + 448 * 2 * U32 * s) / 448, w + " scale")
                each = np.repeat(host(scales[i]), 256)[:len(x)]
                got = oracle.held(codes[i].cpu().numpy(), host(scales[i]))
                within(got, x, np.maximum(2.0 ** -4 * np.abs(x), least * each) * (1 + 2.0 ** -10) + err + 8 * U32 * 448 * each,
                       w + " codes")
            v_codes = self.v[i].cpu().numpy()
            assert np.all((v_codes > 0) == (v > 0)), w + " a second moment held as 0"


SIZES = {
    "one": [1], "block_edges": [255, 256, 257, 1], "chunk_edges": [2047, 2048, 2049, 4096, 8193],
    "empty_ones": [0, 5, 0, 300, 0], "long": [3_000_001, 40], "twentyfive": [100 + 37 * i for i in range(25)],
    "two_launches": [1 + (i * 37) % 400 for i in range(390)],
}
TYPES = {"f32": ("f32", F32), "f32_bf16_grads": ("f32", BF), "bf16": ("bf16", BF), "bf16_f32_grads": ("bf16", F32),
         "masters": ("master", BF), "masters_f32_grads": ("master", F32)}


@pytest.mark.parametrize("eight", [False, True], ids=["32bit", "8bit"])
@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("sizes", SIZES)
def test_one_step(sizes, types, eight):
    kind, grads = TYPES[types]
    c = Case(SIZES[sizes], kind, grads, eight, seed=len(sizes))
    c.run()
    c.check()


@pytest.mark.parametrize("eight", [False, True], ids=["32bit", "8bit"])
@pytest.mark.parametrize("offset", [1, 2, 3, 4, 8])
@pytest.mark.parametrize("kind", ["f32", "bf16", "master"])
def test_any_alignment(kind, offset, eight):
    c = Case([3000, 256, 7], kind, [BF, F32], eight, seed=offset, offset=offset)
    c.run()
    c.check()


@pytest.mark.parametrize("eight", [False, True], ids=["32bit", "8bit"])
@pytest.mark.parametrize("norm,max_norm", [(2.0, 0.5), (2.0, 3.0), (2.0, np.inf), (2.0, 0.0), (0.0, 1.0), (1e20, 1e-10)])
def test_clipping(norm, max_norm, eight):
    c = Case([2000, 9], "f32", F32, eight, norm=norm, max_norm=max_norm)
    c.run()
    c.check()


@pytest.mark.parametrize("hyper", [dict(beta1=0.0), dict(beta2=0.0), dict(weight_decay=0.0), dict(eps=1e-3),
                                   dict(beta1=0.999, beta2=0.99999), dict(lr=0.0), dict(lr=0.5, weight_decay=2.0)],
                         ids=lambda h: "_".join(f"{k}{v}" for k, v in h.items()))
@pytest.mark.parametrize("t", [1, 2, 1000, 2 ** 31 - 1])
def test_parameters_and_step_numbers(hyper, t):
    c = Case([700], "f32", F32, t=t, **hyper)
    c.run()
    c.check()


@pytest.mark.parametrize("eight", [False, True], ids=["32bit", "8bit"])
@pytest.mark.parametrize("kind", ["f32", "bf16", "master"])
def test_steps_from_zeros(kind, eight):
    """Five steps, each from what the one before left: states of zeros, then of its own codes."""
    c = Case([1000, 256, 3], kind, F32, eight, t=1, zeros=True, seed=4)
    gen = torch.Generator(device=dev()).manual_seed(1)
    for t in range(1, 6):
        c.step.fill_(t)
        for g in c.grads:
            g.copy_(torch.randn(g.shape, generator=gen, device=dev()) * 1e-3)
        c.keep()
        c.run()
        c.check(where=f"step {t}")


def test_a_block_without_gradients_stays_zero():
    c = Case([1024], "f32", F32, True, t=1, zeros=True, weight_decay=0.0)
    c.grads[0][256:512] = 0.0
    before = c.params[0].clone()
    c.run()
    c.check()
    assert torch.equal(c.params[0][256:512], before[256:512])
    assert float(c.ms[0][1]) == 0.0 and float(c.vs[0][1]) == 0.0 and not c.m[0][256:512].any()


def test_no_eps():
    """eps 0: with 8-bit states an element that has had no gradient keeps its states of 0 and only
    decays; those beside it step by lr."""
    c = Case([600, 40], "f32", F32, True, t=1, zeros=True, weight_decay=0.5, lr=1e-2, eps=0.0)
    for g in c.grads:
        g[::2] = 0.0
    p = [x.double().clone() for x in c.params]
    c.run()
    c.gd.check()
    for i, g in enumerate(c.grads):
        off = g == 0
        assert not c.m[i][off].any() and not c.v[i][off].any() and bool((c.v[i][~off] > 0).all())
        want = p[i] * (1 - 5e-3) - 1e-2 * g.double().sign()
        assert float((c.params[i].double() - want).abs().max()) <= 64 * U32 * 0.2


def test_small_second_moments():
    """Gradients 2^-30 of their block's largest: sqrt(v) falls below the codes, is held as the
    smallest one, and the next steps move those weights by no more than they should."""
    c = Case([512], "f32", F32, True, t=1, zeros=True, weight_decay=0.0, lr=1e-2)
    c.grads[0].fill_(2.0 ** -30)
    c.grads[0][::256] = 1.0
    for t in range(1, 4):
        c.step.fill_(t)
        before = c.params[0].clone()
        c.run()
        assert bool((c.v[0] > 0).all())
        assert float((c.params[0] - before).abs().max()) <= 1.1e-2
    c.gd.check()


def test_scales_below_the_normal_range_hold_zeros():
    c = Case([256], "f32", F32, True, t=1, zeros=True)
    c.grads[0].fill_(2.0 ** -120)  # g^2 is 0, m below 448 times fp32's least normal value
    c.run()
    assert not c.m[0].any() and not c.v[0].any() and float(c.ms[0]) == 0.0 and float(c.vs[0]) == 0.0


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_bad_gradient(bad):
    """32 bits: its own weight and states. 8 bits: its weight, and its block's states."""
    c = Case([1024], "f32", F32)
    c.grads[0][300] = bad
    c.run()
    for t in (c.params[0], c.m[0], c.v[0]):
        fine = torch.isfinite(t)
        assert int((~fine).sum()) == 1 and not bool(fine[300])
    c = Case([1024], "f32", F32, True)
    c.grads[0][300] = bad
    c.run()
    assert torch.isnan(c.params[0][300]) and int(torch.isfinite(c.params[0]).sum()) == 1023
    c.run()
    bad_now = ~torch.isfinite(c.params[0])
    assert not bool(bad_now[:256].any()) and not bool(bad_now[512:].any())


def test_a_norm_that_is_not_a_number():
    c = Case([300], "f32", F32, norm=float("nan"), max_norm=1.0)
    c.run()
    assert bool(torch.isnan(c.params[0]).all())


def test_step_numbers_below_one_count_as_one():
    from paper_2608_02625_gb300 import binding as B
    B.device_error(clear=True)
    for t in (0, -5):
        c = Case([300], "f32", F32, t=t)
        c.run()
        c.check(t=1)
        assert B.device_error(clear=True) == 1  # DLM_DEVERR_LENGTH


def test_tuples_ranks_and_empty_lists():
    from paper_2608_02625_gb300 import binding as B
    c = Case([24], "bf16", BF)
    shaped = [[x.view(2, 3, 4) for x in t] for t in (c.params, c.grads, c.m, c.v)]
    B.dlm_adamw(tuple(shaped[0]), None, *[tuple(x) for x in shaped[1:]], None, None, c.call_hyper)
    c.check()
    B.dlm_adamw([], None, [], [], [], None, None, c.call_hyper)


def test_captured_steps_follow_their_scalars():
    """A captured step replayed: its number, rate and norm are read as it runs."""
    from paper_2608_02625_gb300 import binding as B
    c = Case([5000, 256], "master", BF, True, t=1, zeros=True, norm=1.0, max_norm=0.5)
    B.device_error(clear=True)  # sets the device up
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            c.run()
    torch.cuda.synchronize()
    for t, lr, norm in ((1, 1e-2, 1.0), (2, 5e-3, 0.25), (7, 1e-3, 4.0)):
        c.step.fill_(t)
        c.lr.fill_(lr)
        c.norm.fill_(norm)
        c.keep()
        graph.replay()
        c.check(where=f"replay {t}")


def test_two_streams():
    cases = [Case([400_000, 77], "f32", BF, eight, seed=3) for eight in (False, True)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    for c, s in zip(cases, streams):
        with torch.cuda.stream(s):
            c.run()
    torch.cuda.synchronize()
    for c in cases:
        c.check()


def test_follows_a_norm_without_waits():
    """The norm of the gradients and the step that clips by it, one after the other."""
    from paper_2608_02625_gb300 import binding as B
    c = Case([300_000, 2000, 5], "master", [BF, F32], norm=0.0, max_norm=0.05)
    ws = torch.empty(B.dlm_clip_grad_norm_workspace_bytes(), dtype=U8, device=dev())
    torch.cuda.synchronize()
    B.dlm_clip_grad_norm(c.grads, None, c.max_norm, c.norm, ws)
    c.run()
    torch.cuda.synchronize()
    want = np.sqrt(sum((host(g) ** 2).sum() for g in c.grads))
    assert abs(float(c.norm) - want) <= 20 * U32 * want
    c.check()


def test_more_than_2_31_elements():
    from paper_2608_02625_gb300 import binding as B
    n = 2 ** 31 + 5000
    gen = torch.Generator(device=dev()).manual_seed(3)
    p = torch.zeros(n, dtype=BF, device=dev())
    g = torch.zeros(n, dtype=BF, device=dev())
    m, v = (torch.zeros(n, dtype=U8, device=dev()) for _ in range(2))
    ms, vs = (torch.zeros((n + 255) // 256, device=dev()) for _ in range(2))
    places = [slice(0, 512), slice(2 ** 31 - 256, 2 ** 31 + 256), slice(n - 136 - 256, n)]
    for s in places:
        p[s] = torch.randn(s.stop - s.start, generator=gen, device=dev()).to(BF)
        g[s] = torch.randn(s.stop - s.start, generator=gen, device=dev()).to(BF)
    before = [host(p[s]) for s in places]
    hyper = B.AdamwParams(lr=torch.full((1,), 0.5, device=dev()), step=torch.ones(1, dtype=torch.int32, device=dev()), **HYPER)
    B.dlm_adamw([p], None, [g], [m], [v], [ms], [vs], hyper)
    torch.cuda.synchronize()
    for s, p0 in zip(places, before):
        want, m1, v1 = oracle.adamw(p0, host(g[s]), 0.0 * p0, 0.0 * p0, 1, 0.5, **HYPER)
        within(host(p[s]), want, HALF[BF] * np.abs(want) + 40 * U32 * (np.abs(p0) + 0.5), f"{s}")
        blocks = slice(s.start // 256, (s.stop + 255) // 256)
        np.testing.assert_allclose(host(ms[blocks]), oracle.block_scales(m1), rtol=8 * U32)
        np.testing.assert_allclose(host(vs[blocks]), oracle.block_scales(np.sqrt(v1)), rtol=8 * U32)
    assert not bool(m[512:2 ** 31 - 256].any())
