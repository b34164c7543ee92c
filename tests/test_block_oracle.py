"""The oracle of the feed-forward block and the optimizer's step, pinned by torch in fp64
and by hand."""
import numpy as np
import pytest
import torch

import oracle


@pytest.mark.parametrize("steps,lr,betas,eps,wd", [(1, 1e-2, (0.9, 0.999), 1e-8, 0.0), (5, 3e-3, (0.8, 0.95), 1e-6, 0.1),
                                                   (3, 1e-1, (0.0, 0.5), 1e-3, 0.5)])
def test_adamw_is_torchs(steps, lr, betas, eps, wd):
    rng = np.random.default_rng(steps)
    p = rng.standard_normal(50)
    t = torch.nn.Parameter(torch.from_numpy(p.copy()))
    opt = torch.optim.AdamW([t], lr=lr, betas=betas, eps=eps, weight_decay=wd)
    m, v = np.zeros(50), np.zeros(50)
    for k in range(1, steps + 1):
        g = rng.standard_normal(50)
        t.grad = torch.from_numpy(g.copy())
        opt.step()
        p, m, v = oracle.adamw(p, g, m, v, k, lr, *betas, eps, wd)
        np.testing.assert_allclose(p, t.detach().numpy(), rtol=1e-12, atol=1e-14)


def test_adamw_by_hand():
    # one step from zeros: m = 0.5 g, v = 0.75 g^2, both corrected back to g and g^2
    p, m, v = oracle.adamw([2.0], [-4.0], [0.0], [0.0], 1, 0.25, 0.5, 0.25, 1.0, 0.5)
    assert m == [-2.0] and v == [12.0] and p == [2.0 - 0.25 - 0.25 * (-4.0 / 5.0)]
    # clipped to half of its size by a norm of 8
    p, m, v = oracle.adamw([2.0], [-4.0], [0.0], [0.0], 1, 0.25, 0.5, 0.25, 1.0, 0.5, norm=8.0 - 1e-6, max_norm=4.0)
    assert np.allclose([m[0], v[0], p[0]], [-1.0, 3.0, 1.75 + 0.25 * 2.0 / 3.0], rtol=1e-14)


def test_e4m3_values_are_torchs():
    want = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(oracle.e4m3_values(), want)
    assert np.nanmax(want) == 448.0 and want[1] == 2.0 ** -9


def test_blocks():
    x = np.zeros(600)
    x[3], x[300], x[599] = -4.48, 44.8, 0.448
    np.testing.assert_allclose(oracle.block_scales(x), [0.01, 0.1, 0.001], rtol=1e-15)
    codes = np.zeros(600, dtype=np.uint8)
    codes[[3, 300, 599]] = [0xFE, 0x7E, 0x7E]
    np.testing.assert_allclose(oracle.held(codes, [0.01, 0.1, 0.001]), x, rtol=1e-15)


def act_of(name, z):
    return {"none": lambda v: v, "silu": torch.nn.functional.silu,
            "gelu": lambda v: torch.nn.functional.gelu(v, approximate="tanh")}[name](z)


@pytest.mark.parametrize("act", ["none", "silu", "gelu"])
def test_activations_are_torchs(act):
    z = torch.linspace(-30, 30, 2001, dtype=torch.float64, requires_grad=True)
    y = act_of(act, z)
    y.sum().backward()
    value, slope = oracle.activation(act, z.detach().numpy())
    np.testing.assert_allclose(value, y.detach().numpy(), rtol=1e-9, atol=1e-13)
    np.testing.assert_allclose(slope, z.grad.numpy(), rtol=1e-9, atol=1e-12)


@pytest.mark.parametrize("act", ["none", "silu", "gelu"])
def test_block_and_gradients_are_autograds(act):
    rng = np.random.default_rng(1)
    t = {n: torch.from_numpy(rng.standard_normal(s)).requires_grad_() for n, s in
         (("x", (7, 16)), ("wg", (24, 16)), ("wu", (24, 16)), ("wd", (16, 24)), ("b", (16,)))}
    gate, up = t["x"] @ t["wg"].T, t["x"] @ t["wu"].T
    h = act_of(act, gate) * up
    h.retain_grad()
    z = h @ t["wd"].T + t["b"]
    y = act_of(act, z) + t["x"]
    dy = rng.standard_normal((7, 16))
    y.backward(torch.from_numpy(dy))
    n = {k: v.detach().numpy() for k, v in t.items()}
    o_h, o_gate, o_up = oracle.gated_linear(n["x"], n["wg"], n["wu"], act)
    o_y, o_z = oracle.linear(o_h, n["wd"], n["b"], act, n["x"])
    np.testing.assert_allclose(o_y, y.detach().numpy(), rtol=1e-11, atol=1e-11)
    dh, dwd, db, _ = oracle.linear_grad(dy, o_h, n["wd"], o_z, act)
    dx, dwg, dwu, _, _ = oracle.gated_linear_grad(dh, n["x"], n["wg"], n["wu"], o_gate, o_up, act, add=dy)
    for got, want in ((dh, h.grad), (dwd, t["wd"].grad), (db, t["b"].grad), (dx, t["x"].grad), (dwg, t["wg"].grad),
                      (dwu, t["wu"].grad)):
        np.testing.assert_allclose(got, want.numpy(), rtol=1e-9, atol=1e-9)
