"""dlm_adamw with 8-bit states and an eps that holds nothing (0, or far below sqrt(v)): second
moments next to and below what fp32 holds.

On the first step, from states of zeros, m / (1 - beta1) = g and sqrt(v / (1 - beta2)) = |g|, so
every weight that has a gradient moves by lr, whatever the gradient's size. In fp32 g^2 and its
product with 1 - beta2 are rounded by half of 2^-149 each where they are below the normal range,
so v is off by at most D = 2^-149, and the quotient's denominator has a floor of 2^-74 times the
correction of sqrt(v): with r = sqrt(1 - beta2) |g| the change is at least r / (sqrt(r^2 + D) +
2^-74) times lr, and at most lr: where r^2 <= D the floor alone is above r, and elsewhere r is
below sqrt(r^2 - D) + 2^-74 too (with x = r^2 / D - 1 >= 0, sqrt(1 + x) < sqrt(x) + sqrt(2)).
Beside that come the roundings of the step itself: 64 U, as in the tests of ordinary gradients."""
import numpy as np
import pytest
import torch

import oracle
from train_util import U32, Guarded, dev, host, within

pytestmark = pytest.mark.gpu

F32, U8 = torch.float32, torch.uint8
LR = 1e-2


class Held:
    """Weights of 0 and states of zeros in 8 bits."""

    def __init__(self, grads, **hyper):
        from paper_2608_02625_gb300 import binding as B
        self.hyper = {**dict(beta1=0.9, beta2=0.95, eps=0.0, weight_decay=0.0), **hyper}
        n, self.gd = len(grads), Guarded()
        zeros = lambda dt, k=n: self.gd.like(torch.zeros(k, dtype=dt, device=dev()))  # noqa: E731
        self.p, self.m, self.v, self.ms, self.vs = zeros(F32), zeros(U8), zeros(U8), zeros(F32, -(-n // 256)), zeros(F32, -(-n // 256))
        self.g = torch.tensor(grads, dtype=F32, device=dev())
        self.step = torch.ones(1, dtype=torch.int32, device=dev())
        self.call = B.AdamwParams(torch.full((1,), LR, device=dev()), self.step, **self.hyper)

    def run(self):
        from paper_2608_02625_gb300 import binding as B
        before = host(self.p)
        B.dlm_adamw([self.p], None, [self.g], [self.m], [self.v], [self.ms], [self.vs], self.call)
        self.gd.check()
        return host(self.p) - before


SIZES = [1e-17, 1e-18, 3e-19, 1e-19, 4e-20, 1e-20, 1e-21, 3e-22, 1e-22, 3e-23, 1e-23, 1e-26, 1e-30]


@pytest.mark.parametrize("beta2", [0.95, 0.999, 0.0])
@pytest.mark.parametrize("n", [1, 256, 777])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_a_first_step_is_lr(size, n, beta2):
    rng = np.random.default_rng(n)
    g = (size * rng.uniform(0.5, 2.0, n) * rng.choice([-1.0, 1.0], n)).astype(np.float32)
    h = Held(g, beta2=beta2)
    moved = h.run()
    g = g.astype(np.float64)
    r2, lost, floor = (1 - beta2) * g * g, 2.0 ** -149, 2.0 ** -74
    low, slack = np.sqrt(r2) / (np.sqrt(r2 + lost) + floor), 64 * U32
    step = moved / (-LR * np.sign(g))
    assert np.all(step >= low * (1 - slack)) and np.all(step <= 1 + slack), (step.min(), step.max())
    # a root that fp32 can tell from 0 is held as a code above 0
    assert bool((h.v.cpu() > 0).numpy()[r2 > 2 * lost].all())


@pytest.mark.parametrize("eps", [1e-25, 1e-12])
@pytest.mark.parametrize("size", [1e-19, 1e-22])
def test_an_eps_above_the_floor_counts(size, eps):
    """The change is lr |g| / (|g| + eps), with |g| off as above and the floor where eps is below it."""
    g = np.full(300, size, dtype=np.float32)
    h = Held(g, beta2=0.95)
    h.call.eps = eps
    moved = h.run()
    x, root = float(g[0]), np.sqrt(0.05)
    lost = 2.0 ** -149
    worst = [np.sqrt(max(0.05 * x * x + s * lost, 0.0)) / root for s in (1, -1)]
    least = x / (worst[0] + max(eps, 2.0 ** -74 / root))
    most = x / (worst[1] + max(eps, 2.0 ** -74 / root))
    within(-moved / LR, np.full(300, (least + most) / 2), (most - least) / 2 + 64 * U32 * most)


def test_steps_that_follow_stay_small():
    """Ten steps of gradients of 1e-19 to 1e-23, some of them 0. A step of these betas is at most 1.02
    lr (Cauchy-Schwarz over the gradients so far, with the corrections). A code next to 0 may be
    twice its m, and two thirds of its sqrt(v); a v next to 2^-149 loses up to a third of itself: below
    1.02 x 2 x 1.5 x 1.25 lr."""
    rng = np.random.default_rng(5)
    n = 600
    h = Held(np.zeros(n, dtype=np.float32), beta2=0.95)
    for t in range(1, 11):
        g = 10.0 ** rng.uniform(-23, -19, n) * rng.choice([-1.0, 0.0, 1.0], n)
        h.g.copy_(torch.from_numpy(g.astype(np.float32)))
        h.step.fill_(t)
        moved = h.run()
        assert np.all(np.isfinite(moved)) and np.abs(moved).max() <= 3.9 * LR, t
    assert bool(torch.isfinite(h.p).all())


def test_a_block_of_all_sizes():
    """Gradients of 1 down to 1e-38 in one block: the small ones' codes are the smallest, and no
    first step is above lr."""
    g = (10.0 ** -np.linspace(0, 38, 256)).astype(np.float32)
    h = Held(g, beta2=0.95)
    moved = h.run()
    assert np.all(moved <= 0) and np.abs(moved).max() <= LR * (1 + 64 * U32)
    ordinary = 0.05 * g.astype(np.float64) ** 2 >= 2.0 ** -126
    r = np.sqrt(0.05) * g.astype(np.float64)
    np.testing.assert_allclose(-moved[ordinary] / LR, (r / (r + 2.0 ** -74))[ordinary], rtol=64 * U32)
    assert bool((h.v.cpu() > 0).numpy()[ordinary].all())
    want = oracle.block_scales(r)
    np.testing.assert_allclose(host(h.vs), want, rtol=16 * U32)
