"""A training step on sampled answers, all its calls in a row: tokens from the logits, their log-probabilities, advantages of
the answers' scores, the policy loss, its gradient with respect to the logits, the norm over it and another parameter's
gradient, and both clipped. Against the float64 oracles from end to end, and captured into a graph."""
from __future__ import annotations

import numpy as np
import pytest

from oracle import losses
from oracle import sampling

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
ANSWERS, LENGTH, VOCAB, GROUP = 24, 10, 1000, 8


@pytest.fixture(scope="module")
def T():
    import paper_1212_2287_amd as T
    T.load_library()
    return T


def _inputs(seed):
    import torch
    rng = np.random.default_rng(seed)
    x = torch.from_numpy(rng.normal(0, 2, (ANSWERS * LENGTH, VOCAB)).astype(np.float32)).cuda()
    other = torch.from_numpy(rng.normal(0, 0.01, (37, 65))).to(torch.bfloat16).cuda()
    return x, other, torch.from_numpy(rng.random(ANSWERS * LENGTH)).cuda()


def _offsets():
    import torch
    return (torch.arange(0, ANSWERS * LENGTH + 1, LENGTH, device="cuda"), torch.arange(0, ANSWERS + 1, GROUP, device="cuda"))


def _step(T, x, other, uniform, sequences, groups, limit, **cut):
    """(tokens, scores, norm, the clipped gradients); an answer's score is how many of its tokens are even."""
    tokens, old_logp, log_kept = T.tree_ens_sample(x, uniform, **cut)
    scores = (1 - tokens % 2).view(ANSWERS, LENGTH).sum(1).float()
    logp, _, stats = T.tree_ens_token_logp(x, tokens)
    advantages = T.tree_ens_group_advantage(scores, groups)
    _, _, grad = T.tree_ens_policy_loss(logp, old_logp, advantages, sequences, flags=T.TREE_ENS_SEQ_MEAN, grad_scale=1.0 / ANSWERS)
    grads = [T.tree_ens_token_logp_backward(x, tokens, stats, grad), other.clone()]
    norm = T.tree_ens_grad_norm(grads)
    return tokens, scores, norm, T.tree_ens_grad_clip(grads, norm, limit)


@pytest.mark.parametrize("limit", [1e-3, 1e3])
@pytest.mark.parametrize("cut", [{}, dict(top_k=40, top_p=0.9), dict(min_p=0.05, scale=1.5)], ids=["all", "top", "min"])
def test_against_the_oracles(T, cut, limit):
    """Of the two log-probabilities in a token's ratio, token_logp's is off by U (4 (1 + |logp| + log S) + V / 256 + 64 + 8),
    below 240 U for logits of +-12 here, the sampler's by 152 U of what is not kept and U |logp|, below 180 U. With the 8 U of
    exp, the advantage's, the share's and the product's roundings a token's gradient is off by less than 440 U of itself, the
    logits' probabilities by U (8 + 6 |z| + 4 log S) and the 8 U of their own product, below 200 U: 700 U together, with room.
    At another scale than 1 the ratio is not 1: no token's may lie where it could fall on either side of the clip's edge."""
    x, other, uniform = _inputs(3)
    sequences, groups = _offsets()
    tokens, scores, norm, clipped = _step(T, x, other, uniform, sequences, groups, limit, **cut)

    h = x.double().cpu().numpy()
    want, old, _ = sampling.sample(h, uniform.cpu().numpy(), **cut)
    assert np.array_equal(tokens.cpu().numpy(), want)
    score = (want % 2 == 0).reshape(ANSWERS, LENGTH).sum(1)
    assert np.array_equal(scores.cpu().numpy(), score)
    advantages = losses.group_advantage(score, groups.cpu().numpy(), 1e-6)
    logp, _, stats = losses.token_logp(h, want)
    ratio = np.exp(logp - old)
    assert (np.abs(ratio - 0.8) > 1e-4).all() and (np.abs(ratio - 1.2) > 1e-4).all()
    _, _, g = losses.policy_loss(logp, old, advantages, sequences.cpu().numpy(), mean=True, grad_scale=1.0 / ANSWERS)
    grad = losses.token_logp_grad(h, want, g)
    p = np.exp(h - h.max(1, keepdims=True) - stats[:, 1:])
    bound = 700 * U * np.abs(g)[:, None] * (p + (np.arange(VOCAB) == want[:, None]))
    o = other.double().cpu().numpy()
    total = np.sqrt((grad ** 2).sum() + (o ** 2).sum())
    off = np.sqrt((bound ** 2).sum()) + (U + 2.0 ** -40) * total
    assert abs(norm.item() - total) <= off
    factor = min(1.0, limit / (total + 1e-6))
    rel = 5 * U + off / total
    assert (np.abs(clipped[0].double().cpu().numpy() - grad * factor) <= factor * bound + rel * np.abs(grad) * factor + 2.0 ** -126).all()
    assert (np.abs(clipped[1].double().cpu().numpy() - o * factor) <= (rel + 2.0 ** -8) * np.abs(o) * factor + 2.0 ** -126).all()


def test_captured_into_a_graph(T):
    """Steps that change their own logits, replayed with new random numbers between eager work: as eager ones, bit for bit."""
    import torch
    x, other, uniform = _inputs(4)
    sequences, groups = _offsets()

    def step(x, uniform):
        tokens, scores, norm, clipped = _step(T, x, other, uniform, sequences, groups, 0.05, top_p=0.95)
        x -= 20.0 * clipped[0]
        return tokens, scores, norm, clipped

    eager = x.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(x.clone(), uniform)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tokens, scores, norm, clipped = step(x, uniform)
    rng = np.random.default_rng(5)
    for k in range(5):
        uniform.copy_(torch.from_numpy(rng.random(uniform.numel())))
        want = step(eager, uniform)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = (tokens, scores, norm, clipped)
        assert all(torch.equal(a, b) for a, b in zip(got[:3], want[:3])), k
        assert all(torch.equal(a, b) for a, b in zip(got[3], want[3])) and torch.equal(x, eager), k
    assert not torch.equal(x, _inputs(4)[0])
