"""A generator learns from the scores of a tree ensemble.

The ensemble plays the reward model: it scores sampled answers from features of theirs (here, which tokens an
answer holds). The generator is the smallest there is, a table of logits for each position of an answer, so that
everything else on the path is what a real program runs: answers are sampled from the logits, scored and the best of
every prompt kept (predict_topk), the log-probabilities of their tokens are taken from the logits, a policy loss on
group-relative advantages and a preference loss on the order of the scores are computed with their gradients, the
gradients go back through the logits and are clipped by their norm.

    python examples/learn_from_scores.py
"""
from __future__ import annotations

import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1212_2287_amd as T  # noqa: E402

PROMPTS, ANSWERS, LENGTH, VOCAB = 32, 8, 24, 136


def reward_model(seed: int = 0) -> "T.TreeEnsemble":
    """One stump for each token: answers that hold it gain (or lose) its value."""
    value = np.random.default_rng(seed).standard_normal(VOCAB).astype(np.float32)
    leaf = np.stack([np.zeros(VOCAB, np.float32), np.zeros(VOCAB, np.float32), value], 1).ravel()
    one = lambda root, left, right: np.tile(np.array([root, left, right]), VOCAB)  # noqa: E731
    feature = one(0, -1, -1)
    feature[::3] = np.arange(VOCAB)
    return T.TreeEnsemble.from_arrays(np.arange(VOCAB + 1) * 3, feature, one(0.5, 0, 0), one(1, -1, -1), one(2, -1, -1), leaf)


def train(steps: int = 30, rate: float = 8.0, max_norm: float = 1.0, loss: str = "policy", seed: int = 0) -> list[float]:
    """The mean score of the answers at each step. `loss`: "policy" or "preference"."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    table = torch.zeros(LENGTH, VOCAB, device="cuda")
    start = table.clone()  # the reference policy
    n_answers = PROMPTS * ANSWERS
    groups = torch.arange(0, n_answers + 1, ANSWERS, device="cuda")
    sequences = torch.arange(0, n_answers * LENGTH + 1, LENGTH, device="cuda")
    position = torch.arange(LENGTH, device="cuda").repeat(n_answers)
    history = []
    with reward_model(seed) as model:
        for _ in range(steps):
            logits = table[position]
            uniform = torch.rand(n_answers * LENGTH, device="cuda", dtype=torch.float64, generator=g)
            tokens, old_logp, _ = T.tree_ens_sample(logits, uniform)
            held = torch.zeros(n_answers, VOCAB, device="cuda")
            held.scatter_(1, tokens.view(n_answers, LENGTH), 1.0)
            scores, best, _ = model.predict_topk(held, groups, 1)
            history.append(float(scores.mean()))

            logp, _, stats = T.tree_ens_token_logp(logits, tokens)
            ref_logp, _, _ = T.tree_ens_token_logp(start[position], tokens)
            if loss == "policy":
                advantages = T.tree_ens_group_advantage(scores, groups)
                _, _, grad = T.tree_ens_policy_loss(logp, old_logp, advantages, sequences, ref_logp=ref_logp, kl_coef=0.01,
                                                    flags=T.TREE_ENS_SEQ_MEAN, grad_scale=1.0 / n_answers)
            else:
                _, _, grad = T.tree_ens_preference_loss(logp, sequences, scores, groups, ref_logp=ref_logp, beta=1.0,
                                                        flags=T.TREE_ENS_SEQ_MEAN, grad_scale=1.0 / PROMPTS)
            grad_logits = T.tree_ens_token_logp_backward(logits, tokens, stats, grad, grad_logits=logits)
            grad_table = torch.zeros_like(table).index_add_(0, position, grad_logits)
            T.tree_ens_grad_clip([grad_table], T.tree_ens_grad_norm([grad_table]), max_norm)
            table -= rate * LENGTH * grad_table
    return history


if __name__ == "__main__":
    for name in ("policy", "preference"):
        scores = train(loss=name)
        print(f"{name}: mean score of an answer " + " ".join(f"{s:.2f}" for s in scores[::5] + scores[-1:]))
