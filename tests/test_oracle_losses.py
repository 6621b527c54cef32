"""The float64 oracle of the losses against torch's autograd, differences and hand-worked values."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from oracle import losses as O


@pytest.mark.parametrize("scale", [1.0, 0.7])
def test_token_logp_and_gradient_against_autograd(scale):
    rng = np.random.default_rng(0)
    x = rng.normal(0, 3, (5, 17))
    x[1, 3:9] = -np.inf
    t = np.array([0, 1, 16, -100, 17])
    g, h = rng.normal(size=5), rng.normal(size=5)
    y = torch.tensor(x, requires_grad=True)
    lp = torch.log_softmax(scale * y, 1)
    live = torch.tensor((t >= 0) & (t < 17))
    at = lp[torch.arange(5), torch.tensor(np.where(live, t, 0))]
    ent = -(lp.exp() * lp.masked_fill(lp == -torch.inf, 0.0)).sum(1)
    # autograd of masked entries is 0 * inf: their rows are checked by differences below
    logp, entropy, stats = O.token_logp(x, t, scale)
    assert np.allclose(logp, torch.where(live, at, 0.0).detach(), rtol=1e-13, atol=1e-13)
    assert np.allclose(entropy, torch.where(live, ent, 0.0).detach(), rtol=1e-12, atol=1e-13)
    assert np.allclose(stats[:3, 0], x[:3].max(1)) and not stats[3:].any()
    rows = torch.tensor([0, 2])
    (torch.tensor(g)[rows] * at[rows] + torch.tensor(h)[rows] * ent[rows]).sum().backward()
    grad = O.token_logp_grad(x, t, g, h, scale)
    assert np.allclose(grad[[0, 2]], y.grad[[0, 2]], rtol=1e-11, atol=1e-13)
    assert not grad[3:].any() and not grad[1, 3:9].any()
    for v in (0, 1, 12):
        def f(e):
            z = x.copy()
            z[1, v] += e
            a, b, _ = O.token_logp(z, t, scale)
            return g[1] * a[1] + h[1] * b[1]
        assert abs((f(1e-5) - f(-1e-5)) / 2e-5 - grad[1, v]) < 1e-8


def test_token_logp_of_a_row_without_anything():
    logp, entropy, stats = O.token_logp(np.full((1, 4), -np.inf), [2])
    assert logp[0] == -np.inf and entropy[0] == 0 and stats[0].tolist() == [-np.inf, 0.0]
    assert not O.token_logp_grad(np.full((1, 4), -np.inf), [2], [1.0], [1.0]).any()


def _random_sequences(rng):
    seqs = np.concatenate([[0], np.cumsum([3, 0, 1, 5, 2, 4, 2])])
    groups = np.array([0, 2, 2, 6, 7])
    n = int(seqs[-1])
    return seqs, groups, -rng.exponential(size=n), -rng.exponential(size=n), rng.random(n) < 0.7


@pytest.mark.parametrize("mean", [False, True])
@pytest.mark.parametrize("masked", [False, True])
def test_preference_loss_gradient_by_differences(mean, masked):
    rng = np.random.default_rng(3)
    seqs, groups, lp, ref, mask = _random_sequences(rng)
    mask = mask if masked else None
    scores = np.array([1.0, 0.0, 2.0, 2.0, 3.0, np.nan, 1.0])
    args = dict(ref_logp=ref, mask=mask, beta=0.7, smoothing=0.1, mean=mean)
    loss, h, grad = O.preference_loss(lp, seqs, scores, groups, grad_scale=1.5, **args)
    assert loss[1] == 0 and loss[3] == 0 and loss[0] > 0 and loss[2] > 0
    assert not grad[seqs[6]:].any() and not grad[seqs[5]:seqs[6]].any()
    for t in range(len(lp)):
        def f(e):
            z = lp.copy()
            z[t] += e
            return 1.5 * O.preference_loss(z, seqs, scores, groups, **args)[0].sum()
        assert abs((f(1e-6) - f(-1e-6)) / 2e-6 - grad[t]) < 1e-8


def test_preference_loss_of_one_pair_by_hand():
    # h = 0.5 * (-1 - -2, -3 - -2.5) = (0.5, -0.25); d = 0.75
    loss, h, grad = O.preference_loss([-1.0, -3.0], [0, 1, 2], [5.0, 4.0], [0, 2], ref_logp=[-2.0, -2.5], beta=0.5)
    assert np.allclose(h, [0.5, -0.25])
    assert np.allclose(loss, np.log(1 + np.exp(-0.75)))
    assert np.allclose(grad, np.array([-1, 1]) * 0.5 / (1 + np.exp(0.75)))


@pytest.mark.parametrize("mean", [False, True])
@pytest.mark.parametrize("masked", [False, True])
def test_policy_loss_gradient_by_differences(mean, masked):
    rng = np.random.default_rng(5)
    seqs, _, lp, ref, mask = _random_sequences(rng)
    old = lp - rng.normal(0, 0.3, len(lp))
    adv = np.array([1.0, 2.0, -1.5, 0.5, -0.5, 0.0, 2.0])
    args = dict(ref_logp=ref, mask=mask if masked else None, clip_low=0.1, clip_high=0.2, kl_coef=0.3, mean=mean)
    loss, kl, grad = O.policy_loss(lp, old, adv, seqs, grad_scale=0.5, **args)
    assert (kl >= 0).all() and loss[1] == 0 and kl[1] == 0
    for t in range(len(lp)):
        def f(e):
            z = lp.copy()
            z[t] += e
            return 0.5 * O.policy_loss(z, old, adv, seqs, **args)[0].sum()
        assert abs((f(1e-7) - f(-1e-7)) / 2e-7 - grad[t]) < 1e-6


def test_policy_loss_of_single_tokens_by_hand():
    # ratio 2: gain clipped at 1.2 for A = 1 (no gradient), not for A = -1
    lp, old = [np.log(2.0), np.log(2.0)], [0.0, 0.0]
    loss, kl, grad = O.policy_loss(lp, old, [1.0, -1.0], [0, 1, 2])
    assert np.allclose(loss, [-1.2, 2.0]) and np.allclose(grad, [0.0, 2.0]) and not kl.any()


def test_group_advantage_by_hand():
    a = O.group_advantage([1.0, 3.0, 7.0, 9.0], [0, 2, 3], eps=1.0)
    assert np.allclose(a, [-0.5, 0.5, 0.0, 0.0])
    assert np.allclose(O.group_advantage([1.0, 3.0], [0, 2], 1.0, center_only=True), [-1.0, 1.0])
