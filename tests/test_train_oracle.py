"""Pins of the oracle of training the refiner's last layer (oracle/train.py): torch's
autograd in fp64, differences, closed forms and hand-worked values."""
import numpy as np
import pytest
import torch

import oracle


def rng(seed):
    return np.random.default_rng(seed)


@pytest.mark.parametrize("N,d", [(1, 1), (3, 5), (7, 64)])
def test_layer_norm_and_gradients_against_autograd(N, d):
    g = rng(N * 100 + d)
    x, w, b, dy = g.normal(1.0, 2.0, (N, d)), g.normal(1, 0.3, d), g.normal(0, 0.3, d), g.normal(size=(N, d))
    tx, tw, tb = (torch.tensor(v, requires_grad=True) for v in (x, w, b))
    ref = torch.nn.functional.layer_norm(tx, (d,), tw, tb, 1e-5)
    ref.backward(torch.tensor(dy))
    out, mean, rstd = oracle.layer_norm(x, w, b, 1e-5)
    np.testing.assert_allclose(out, ref.detach().numpy(), rtol=1e-10, atol=1e-12)
    for got, want in zip(oracle.layer_norm_grad(dy, x, w, mean, rstd), (tx.grad, tw.grad, tb.grad)):
        np.testing.assert_allclose(got, want.numpy(), rtol=1e-8, atol=1e-9)


def test_layer_norm_hand_worked():
    # mean 3, variance 4 (deviations -2, +2): xhat = -1, +1 at eps = 0
    out, mean, rstd = oracle.layer_norm([[1.0, 5.0]], [2.0, 3.0], [0.5, -0.5], 0.0)
    assert mean[0] == 3.0 and rstd[0] == 0.5
    np.testing.assert_array_equal(out, [[-1.5, 2.5]])


def loss_case(seed, N=6, V=11, d=5):
    g = rng(seed)
    t = g.integers(0, V, N)
    t[1], t[-1] = -1, V  # not scored
    return g.normal(size=(N, d)), g.normal(size=(V, d)), t, g.uniform(0.1, 2.0, N)


def test_loss_and_gradients_against_autograd():
    h, w, t, dl = loss_case(3)
    th, tw = (torch.tensor(v, requires_grad=True) for v in (h, w))
    on = torch.tensor((t >= 0) & (t < len(w)))
    ref = torch.nn.functional.cross_entropy(th @ tw.T, torch.where(on, torch.tensor(t), -100), reduction="none")
    (ref * torch.tensor(dl)).sum().backward()
    loss, lse = oracle.lm_head_loss(h, w, t)
    np.testing.assert_allclose(loss, ref.detach().numpy(), rtol=1e-12, atol=1e-12)
    assert loss[1] == lse[1] == loss[-1] == lse[-1] == 0.0
    dh, dw, _ = oracle.lm_head_loss_grad(h, w, t, lse, dl)
    np.testing.assert_allclose(dh, th.grad.numpy(), rtol=1e-11, atol=1e-12)
    np.testing.assert_allclose(dw, tw.grad.numpy(), rtol=1e-11, atol=1e-12)
    assert np.all(dh[1] == 0) and np.all(dh[-1] == 0)


def test_loss_gradients_against_differences():
    h, w, t, dl = loss_case(4)
    _, lse = oracle.lm_head_loss(h, w, t)
    dh, dw, _ = oracle.lm_head_loss_grad(h, w, t, lse, dl)
    step = 1e-6
    total = lambda h, w: float((oracle.lm_head_loss(h, w, t)[0] * dl).sum())  # noqa: E731
    for a, grad in ((h, dh), (w, dw)):
        for i in np.ndindex(a.shape):
            up, down = a.copy(), a.copy()
            up[i] += step
            down[i] -= step
            diff = (total(up, w) - total(down, w)) if a is h else (total(h, up) - total(h, down))
            assert abs(diff / (2 * step) - grad[i]) < 1e-7


def test_loss_hand_worked():
    # logits ln 1, ln 2, ln 5: the probability of the second is 1/4
    loss, lse = oracle.lm_head_loss([[1.0]], np.log([[1.0], [2.0], [5.0]]), [1])
    np.testing.assert_allclose([loss[0], lse[0]], [np.log(4.0), np.log(8.0)], rtol=1e-14)


def test_clip_against_torch_and_by_hand():
    outs, norm = oracle.clip_grad_norm([[3.0], [4.0, 0.0]], 1.0)
    assert norm == 5.0
    np.testing.assert_allclose(np.concatenate(outs), [0.6, 0.8, 0.0], rtol=1e-6)
    outs, norm = oracle.clip_grad_norm([[3.0], [4.0]], 6.0)
    assert norm == 5.0 and outs[0][0] == 3.0 and outs[1][0] == 4.0
    g = rng(9)
    ps = [torch.tensor(g.normal(size=n), requires_grad=True) for n in (3, 100, 17)]
    for p in ps:
        p.grad = torch.tensor(g.normal(size=p.shape))
    grads = [p.grad.numpy().copy() for p in ps]
    ref = torch.nn.utils.clip_grad_norm_(ps, 0.7)
    outs, norm = oracle.clip_grad_norm(grads, 0.7)
    np.testing.assert_allclose(norm, float(ref), rtol=1e-12)
    for o, p in zip(outs, ps):
        np.testing.assert_allclose(o, p.grad.numpy(), rtol=1e-12)
