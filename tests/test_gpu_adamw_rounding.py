"""What dlm_adamw holds, bit for bit: every product and sum of m and v is rounded to fp32 by itself, in
the order of the formula, so that 32-bit states are those of the same operations one by one, and 8-bit
codes of m and their scales too (the codes of sqrt(v) but for roots next to a border: theirs is an
approximation, and so are scales next to one)."""
import pytest
import torch

from train_util import dev

pytestmark = pytest.mark.gpu

BF, F32, U8 = torch.bfloat16, torch.float32, torch.uint8
N = 2_000_003
BETA1, BETA2 = 0.9, 0.95


def scalar(x):
    return torch.tensor(x, dtype=F32, device=dev())


def moments(g, m, v, clip):
    x = g.float() * scalar(clip)
    m = m * scalar(BETA1) + x * scalar(1.0 - BETA1)
    return m, v * scalar(BETA2) + (x * x) * scalar(1.0 - BETA2)


def run(p, g, m, v, ms, vs, clip):
    from paper_2608_02625_gb300 import binding as B
    # clip (1 + 1e-6) / (norm + 1e-6), rounded to fp32: clip
    norm = torch.full((1,), 1.0, device=dev())
    h = B.AdamwParams(torch.full((1,), 1e-3, device=dev()), torch.full((1,), 5, dtype=torch.int32, device=dev()), BETA1, BETA2, 1e-8, 0.1,
                      norm, clip * (1.0 + 1e-6))
    B.dlm_adamw([p], None, [g], [m], [v], ms, vs, h)


def inputs(seed, dtype):
    gen = torch.Generator(device=dev()).manual_seed(seed)
    r = lambda std: torch.empty(N, device=dev()).normal_(0.0, std, generator=gen)  # noqa: E731
    return r(0.02), r(1e-3).to(dtype), r(3e-4), r(1e-3).square_().add_(1e-10)


@pytest.mark.parametrize("grads", [BF, F32])
@pytest.mark.parametrize("clip", [1.0, 0.5, 0.37])
@pytest.mark.parametrize("offset", [0, 1])
def test_states_in_32_bits(grads, clip, offset):
    p, g, m, v = (t[offset:] for t in inputs(1, grads))
    want = moments(g, m, v, clip)
    run(p, g, m, v, None, None, clip)
    assert torch.equal(m, want[0]) and torch.equal(v, want[1])


def blocks(x):
    return torch.nn.functional.pad(x, (0, -len(x) % 256)).view(-1, 256)


def codes(x, above_zero):
    s = blocks(x).abs().amax(1) * scalar(1.0 / 448.0)
    q = (blocks(x) * (1.0 / s)[:, None]).to(torch.float8_e4m3fn).view(U8).reshape(-1)[:len(x)]
    return (torch.where((x > 0) & (q == 0), torch.ones_like(q), q) if above_zero else q), s


@pytest.mark.parametrize("grads", [BF, F32])
@pytest.mark.parametrize("clip", [1.0, 0.37])
def test_states_in_8_bits(grads, clip):
    p, g, m, v = inputs(2, grads)
    (mq, ms), (vq, vs) = codes(m, False), codes(v.sqrt(), True)
    each = lambda s: s.repeat_interleave(256)[:N]  # noqa: E731
    values = lambda q, s: q.view(torch.float8_e4m3fn).float() * each(s)  # noqa: E731
    m1, v1 = moments(g, values(mq, ms), values(vq, vs).square(), clip)
    (want_mq, want_ms), (want_vq, want_vs) = codes(m1, False), codes(v1.sqrt(), True)
    run(p, g, mq, vq, [ms], [vs], clip)
    assert torch.equal(ms, want_ms) and torch.equal(mq, want_mq)
    # a root is off by one last place at most, a scale by that and its own rounding, and a quotient by
    # both and its own: 5 U of values up to 448, whose borders of codes are 2^-4 of them apart and more
    assert bool(((vs - want_vs).abs() <= 2.0 ** -22 * want_vs).all())
    step = (vq.int() - want_vq.int()).abs()
    assert int(step.max()) <= 1 and int(step.sum()) <= N * 5 * 2.0 ** -24 * 2 ** 4 * 4
