"""The float64 oracle of sampling and clipping against hand-worked values, counting and torch."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from oracle import sampling as O

# weights 1, 1/2, 1/4, 1/8, 1/8 of 2 in all, at the places 3, 0, 4, 1, 2
ROW = np.log([0.5, 0.125, 0.125, 1.0, 0.25])


@pytest.mark.parametrize("params,kept", [
    (dict(), [3, 0, 4, 1, 2]), (dict(top_k=2), [3, 0]), (dict(top_k=4), [3, 0, 4, 1]), (dict(top_k=9), [3, 0, 4, 1, 2]),
    (dict(min_p=0.2), [3, 0, 4]), (dict(min_p=1.0), [3]), (dict(top_p=0.4), [3]), (dict(top_p=0.6), [3, 0]),
    (dict(top_p=0.76), [3, 0, 4]), (dict(top_p=0.95), [3, 0, 4, 1, 2]), (dict(top_p=1e-9), [3]),
    (dict(top_k=2, top_p=0.7), [3, 0]), (dict(top_k=2, top_p=0.6), [3]),  # 1 of 1.5 is two thirds
    (dict(min_p=0.2, top_p=0.6), [3, 0]), (dict(scale=2.0, min_p=0.2), [3, 0]),
])
def test_kept_tokens_by_hand(params, kept):
    assert O.kept_tokens(ROW, **params)[0] == kept


def test_tokens_by_hand():
    # in order of the vocabulary the weights 0.5 .125 .125 1 .25 end at .25, .3125, .375, .875 and 1 of the total
    u = np.array([0.0, 0.2499, 0.2501, 0.3124, 0.3126, 0.3749, 0.3751, 0.8749, 0.8751, 0.9999])
    tokens, logp, log_kept = O.sample(np.tile(ROW, (10, 1)), u)
    assert tokens.tolist() == [0, 0, 1, 1, 2, 2, 3, 3, 4, 4]
    assert np.allclose(logp, ROW[tokens] - np.log(2.0)) and not log_kept.any()
    tokens, logp, log_kept = O.sample(np.tile(ROW, (3, 1)), [0.0, 0.33, 0.34], top_k=2)
    assert tokens.tolist() == [0, 0, 3] and np.allclose(log_kept, np.log(0.75))
    assert np.allclose(logp, ROW[tokens] - np.log(2.0))


def test_rows_of_special_values():
    x = np.array([[0.0, np.nan], [0.0, np.inf], [-np.inf, -np.inf], [-np.inf, 5.0]])
    tokens, logp, log_kept = O.sample(x, np.full(4, 0.99))
    assert tokens.tolist() == [-1, -1, -1, 1]
    assert np.isnan(logp[:2]).all() and logp[2] == -np.inf and logp[3] == 0 and log_kept[2:].tolist() == [0, 0]
    assert O.sample(x[3:], [0.5], scale=0.0)[0] == -1


def test_equals_are_kept_by_index():
    assert O.kept_tokens(np.zeros(6), top_k=3)[0] == [0, 1, 2]
    assert O.kept_tokens(np.zeros(6), top_p=0.5)[0] == [0, 1, 2]
    assert O.kept_tokens(np.zeros(6), min_p=1.0)[0] == list(range(6))


def test_even_random_numbers_give_the_distribution():
    x = np.random.default_rng(0).normal(0, 1, 9)
    n = 20_000
    tokens, _, _ = O.sample(np.tile(x, (n, 1)), (np.arange(n) + 0.5) / n, scale=1.3, top_k=6, top_p=0.9)
    order, w = O.kept_tokens(x, 1.3, 6, 0.9)
    p = np.zeros(9)
    p[order] = w[order] / w[order].sum()
    assert np.abs(np.bincount(tokens, minlength=9) / n - p).max() <= 1.0 / n + 1e-12


def test_norm_and_clipping_against_torch():
    rng = np.random.default_rng(1)
    ts = [rng.normal(size=s) for s in ((3, 4), (7,), (), (0,), (2, 2, 2))]
    params = [torch.nn.Parameter(torch.zeros(t.shape, dtype=torch.float64)) for t in ts]
    for limit in (0.5, 100.0):
        for p, t in zip(params, ts):
            p.grad = torch.tensor(t, dtype=torch.float64)
        norm = torch.nn.utils.clip_grad_norm_(params, limit).item()
        assert abs(O.grad_norm(ts) - norm) < 1e-12
        for p, c in zip(params, O.grad_clip(ts, norm, limit)):
            assert np.allclose(p.grad.numpy(), c, rtol=1e-12, atol=0)
