"""Performance cases of the operators that train a language model on the scores of its answers.

A prompt's sampled answers are a query's candidates: the ensemble scores them, and the generator learns
from the scores. Tokens are packed: sequence s owns tokens [seq_offsets[s], seq_offsets[s + 1]) and
group g owns sequences [group_offsets[g], group_offsets[g + 1]), the offsets that per-query top-k takes.

  logp    log-probabilities (and entropies) of the tokens that were sampled, from logits
  grad    their gradient with respect to the logits
  pref    pairwise preference loss over the pairs that the scores order, with its gradient
  adv     advantages of the scores relative to their group
  policy  clipped policy loss with a KL term, with its gradient

Where `own` is false, `run` computes them by elementary torch operations in 32 bits.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}

# logits: `rows` tokens of a vocabulary of `vocab`, rows `pad` logits further apart than that; `ignored`: share of
# the tokens that do not count (a prompt's), `banned`: share of the vocabulary whose logits are -inf.
_LOGITS = {"rows": 1, "vocab": 32_000, "pad": 0, "dtype": "bf16", "scale": 1.0, "entropy": False, "ignored": 0.0,
           "banned": 0.0}
# candidates: `groups` of `few` to `many`, sequences of `short` to `long` tokens (uniform in the logarithm), a share
# `empty` of them without any; `prompt`: share of a sequence at most that the mask leaves out, 0: no mask.
_SEQS = {"groups": 64, "few": 2, "many": 2, "short": 20, "long": 1_000, "empty": 0.0, "prompt": 0.0, "mean": False}


def _logits(call: str, **changes) -> dict:
    return {"call": call, **_LOGITS, **changes}


def _seqs(call: str, **changes) -> dict:
    return {"call": call, **_SEQS, **changes}


def listed() -> list:
    return [
        # generation: the log-probability and entropy of the one token just sampled
        _logits("logp", name="logp_one_token", rows=1, vocab=128_000, entropy=True),
        # a few drafted tokens are checked, sampled at a temperature, in single precision; an odd vocabulary
        _logits("logp", name="logp_24_f32_odd", rows=24, vocab=50_001, dtype="f32", scale=1.25),
        # a training micro-batch of prompts with answers: the prompts' tokens do not count
        _logits("logp", name="logp_8k_prompted", rows=8_192, vocab=32_000, ignored=0.4),
        # a full training batch of a large vocabulary, with entropies: the largest case
        _logits("logp", name="logp_16k_x_131k", rows=16_384, vocab=131_072, entropy=True),
        # gradient of a short answer, half precision, padded odd rows, part of the vocabulary not allowed
        _logits("grad", name="grad_200_f16_odd", rows=200, vocab=32_001, pad=6, dtype="f16", entropy=True, banned=0.3),
        # gradient of a training micro-batch of a large vocabulary
        _logits("grad", name="grad_4k_x_131k", rows=4_096, vocab=131_072),
        # pairs of a preferred and a rejected answer, with smoothed labels
        _seqs("pref", name="pref_64_pairs", smoothing=0.1),
        # the ranking workload's queries of 20 to 200 candidates: every pair that the scores order
        _seqs("pref", name="pref_909_queries", groups=909, few=20, many=200, short=16, long=512, prompt=0.5, mean=True,
              smoothing=0.0, empty=0.01),
        # advantages of one rollout step
        _seqs("adv", name="adv_512x16", groups=512, few=16, many=16),
        # advantages of a million scored candidates
        _seqs("adv", name="adv_1M", groups=9_090, few=20, many=200),
        # a small policy step: 16 prompts, 4 answers of each
        _seqs("policy", name="policy_64", groups=16, few=4, many=4, short=1, long=500),
        # a large step over long answers: 19 million tokens
        _seqs("policy", name="policy_4k_long", groups=512, few=8, many=8, short=512, long=16_384, prompt=0.3, mean=True),
    ]


def _log_int(rng, lo: float, hi: float) -> int:
    return max(int(lo), min(int(hi), int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng) -> dict:
    call = rng.choice(["logp", "logp", "grad", "grad", "pref", "pref", "adv", "policy", "policy"])
    if call in ("logp", "grad"):
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        vocab = _log_int(rng, 100, 150_000)
        most = 2 ** 31 / (4 if dtype == "f32" else 2) / (2 if call == "grad" else 1)  # logits of a pass
        return _logits(call, rows=_log_int(rng, 1, min(65_536, most // vocab)), vocab=vocab, dtype=dtype,
                       pad=rng.choice([0, 0, rng.randint(1, 64)]), scale=rng.choice([1.0, 1.0, round(rng.uniform(0.5, 2.0), 3)]),
                       entropy=rng.random() < 0.5, ignored=rng.choice([0.0, 0.3, 0.7]), banned=rng.choice([0.0, 0.0, 0.5]))
    if call == "adv":
        many = _log_int(rng, 2, 1_000)
        return _seqs(call, groups=_log_int(rng, 1, 1_000_000 // many), few=rng.choice([1, many]), many=many)
    longest = _log_int(rng, 8, 16_384)
    few, many = sorted(_log_int(rng, 2, 300 if call == "pref" else 64) for _ in range(2))
    tokens = many * longest
    pairs = 4.0e7 / many ** 2 if call == "pref" else 1.0e6
    groups = _log_int(rng, 1, max(2.0, min(20_000, 4.0e7 / tokens, pairs)))
    return _seqs(call, groups=groups, few=few, many=many, short=max(1, longest // rng.choice([1, 4, 30, 1_000])), long=longest,
                 empty=rng.choice([0.0, 0.05]), prompt=rng.choice([0.0, 0.5, 0.9]), mean=rng.random() < 0.5,
                 **({"smoothing": rng.choice([0.0, 0.1])} if call == "pref" else {}))


# ----------------------------------------------------------------------------------------------
# inputs
# ----------------------------------------------------------------------------------------------
_BETA, _CLIP_LOW, _CLIP_HIGH, _KL, _EPS = 0.1, 0.2, 0.28, 0.04, 1e-4


def _random(seed: int) -> torch.Generator:
    return torch.Generator(device="cuda").manual_seed(3 * seed + 2)


def _make_logits(case: dict, seed: int) -> dict:
    g = _random(seed)
    n, V, dtype = case["rows"], case["vocab"], _DTYPES[case["dtype"]]
    wide = torch.empty((n, V + case["pad"]), dtype=dtype, device="cuda")
    x = wide[:, :V]
    x.normal_(0.0, 2.5, generator=g)
    t = torch.randint(0, V, (n,), generator=g, device="cuda")
    if case["banned"]:
        x.masked_fill_(torch.rand(V, generator=g, device="cuda") < case["banned"], -math.inf)
    x.scatter_(1, t[:, None], torch.empty((n, 1), device="cuda").normal_(6.0, 4.0, generator=g).to(dtype))
    t.masked_fill_(torch.rand(n, generator=g, device="cuda") < case["ignored"], -100)
    made = {"logits": x, "targets": t, "scale": case["scale"], "entropy": case["entropy"]}
    if case["call"] == "grad":
        # what the losses hand back: nothing for a tenth of the tokens (clipped ones)
        made["grad_logp"] = torch.randn(n, generator=g, device="cuda")
        made["grad_logp"].masked_fill_(torch.rand(n, generator=g, device="cuda") < 0.1, 0.0)
        made["grad_entropy"] = 0.1 * torch.randn(n, generator=g, device="cuda") if case["entropy"] else None
    return made


def _lengths(case: dict, seed: int):
    """Offsets of the groups and of the sequences: the case says which sizes there are, the seed their order."""
    rng, order = np.random.default_rng([case["groups"], case["many"], case["long"]]), np.random.default_rng([seed, 5])
    sizes = order.permutation(rng.integers(case["few"], case["many"] + 1, case["groups"]))
    groups = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int64)
    S = int(groups[-1])
    n = np.rint(np.exp(rng.uniform(math.log(case["short"]), math.log(case["long"]), S))).astype(np.int64)
    n[rng.random(S) < case["empty"]] = 0
    return groups, np.concatenate([[0], np.cumsum(order.permutation(n))]).astype(np.int64)


def _make_seqs(case: dict, seed: int) -> dict:
    g = _random(seed)
    groups, seqs = _lengths(case, seed)
    S = len(seqs) - 1
    made = {"groups": torch.from_numpy(groups).cuda(), "largest": int(np.max(np.diff(groups))),
            # sums of few leaves: equal scores are common
            "scores": torch.empty(S, device="cuda").normal_(generator=g).mul_(8).round_().div_(8)}
    if case["call"] == "adv":
        return made
    N, lens = int(seqs[-1]), torch.from_numpy(np.diff(seqs)).cuda()
    made |= {"seqs": torch.from_numpy(seqs).cuda(), "longest": int(np.max(np.diff(seqs))), "mean": case["mean"]}
    lp = torch.empty(N, device="cuda").exponential_(1.0, generator=g).neg_()
    made["logp"] = lp
    made["ref_logp"] = (lp + torch.empty(N, device="cuda").normal_(0.0, 0.2, generator=g)).clamp_max(-1e-6)
    made["mask"] = None
    if case["prompt"]:
        first = (torch.rand(S, generator=g, device="cuda") * case["prompt"] * lens).long() + made["seqs"][:-1]
        made["mask"] = torch.arange(N, device="cuda") >= first.repeat_interleave(lens, output_size=N)
    if case["call"] == "pref":
        made["smoothing"] = case["smoothing"]
        return made
    # Log ratios to the policy that sampled. The gradient jumps where the ratio passes the clip: ratios that
    # rounding alone would carry over an edge are moved off it.
    r = torch.empty(N, device="cuda").normal_(0.0, 0.15, generator=g)
    low, high = math.log(1 - _CLIP_LOW), math.log(1 + _CLIP_HIGH)
    r = torch.where((r - low).abs() < 1e-4, low - 2e-4, torch.where((r - high).abs() < 1e-4, high + 2e-4, r))
    made["old_logp"] = lp - r
    made["advantages"] = torch.randn(S, generator=g, device="cuda")
    return made


def _make(case: dict, seed: int) -> dict:
    return _make_logits(case, seed) if case["call"] in ("logp", "grad") else _make_seqs(case, seed)


def prepare(case: dict, seed: int) -> dict:
    state = {"call": case["call"], **_make(case, seed)}
    if case["call"] == "grad":  # the forward pass left these
        _, entropy, state["stats"] = _plain_logp({**state, "entropy": True})
        state["entropy_of"] = entropy if case["entropy"] else None
    return state


# ----------------------------------------------------------------------------------------------
# one pass
# ----------------------------------------------------------------------------------------------
def run(state: dict):
    return (_own if own else _plain)[state["call"]](state)


def _own_logp(s):
    import paper_1212_2287_amd as te

    logp, entropy, stats = te.tree_ens_token_logp(s["logits"], s["targets"], scale=s["scale"], want_entropy=s["entropy"])
    return (logp, entropy, stats) if s["entropy"] else (logp, stats)


def _own_grad(s):
    import paper_1212_2287_amd as te

    return te.tree_ens_token_logp_backward(s["logits"], s["targets"], s["stats"], s["grad_logp"], scale=s["scale"],
                                           entropy=s["entropy_of"], grad_entropy=s["grad_entropy"])


def _own_pref(s):
    import paper_1212_2287_amd as te

    return te.tree_ens_preference_loss(s["logp"], s["seqs"], s["scores"], s["groups"], ref_logp=s["ref_logp"], mask=s["mask"],
                                       beta=_BETA, smoothing=s["smoothing"], flags=te.TREE_ENS_SEQ_MEAN if s["mean"] else 0)


def _own_adv(s):
    import paper_1212_2287_amd as te

    return te.tree_ens_group_advantage(s["scores"], s["groups"], eps=_EPS)


def _own_policy(s):
    import paper_1212_2287_amd as te

    return te.tree_ens_policy_loss(s["logp"], s["old_logp"], s["advantages"], s["seqs"], ref_logp=s["ref_logp"], mask=s["mask"],
                                   clip_low=_CLIP_LOW, clip_high=_CLIP_HIGH, kl_coef=_KL,
                                   flags=te.TREE_ENS_SEQ_MEAN if s["mean"] else 0)


def _shifted(s):
    """(z = scale * (x - max), max, row counts) of the logits in 32 bits; a row of -inf alone keeps z = -inf."""
    x, t = s["logits"].float(), s["targets"]
    m = x.amax(1)
    z = (x - torch.where(m == -math.inf, 0.0, m)[:, None]) * s["scale"]
    return z, m, (t >= 0) & (t < x.shape[1])


def _plain_logp(s):
    z, m, live = _shifted(s)
    e = torch.exp(z)
    total = e.sum(1)
    full = live & (total > 0)
    log_sum = torch.log(total)
    at = z.gather(1, torch.where(live, s["targets"], 0)[:, None])[:, 0]
    logp = torch.where(full, at - log_sum, torch.where(live, -math.inf, 0.0))
    stats = torch.stack([torch.where(live, m, 0.0), torch.where(full, log_sum, 0.0)], 1)
    if not s["entropy"]:
        return logp, stats
    entropy = log_sum - torch.where(e > 0, e * z, 0.0).sum(1) / total
    return logp, torch.where(full, entropy, 0.0), stats


def _plain_grad(s):
    z, m, live = _shifted(s)
    z -= s["stats"][:, 1:]
    p = torch.exp(z)
    use = live & (m > -math.inf)
    g = torch.where(use, s["grad_logp"], 0.0)[:, None]
    d = -g * p
    if s["grad_entropy"] is not None:
        h = torch.where(use, s["grad_entropy"], 0.0)[:, None]
        d -= h * p * torch.where(p > 0, z + s["entropy_of"][:, None], 0.0)
    d.scatter_add_(1, torch.where(live, s["targets"], 0)[:, None], g)
    return (d * s["scale"]).to(s["logits"].dtype)


def _padded(offsets, longest: int, n: int):
    """(indices, which are inside) of the segments of `offsets`, one row for each."""
    at = offsets[:-1, None] + torch.arange(longest, device="cuda")
    return at.clamp_max(max(n - 1, 0)), at < offsets[1:, None]


def _counted(s):
    """(indices, which count, divisor) of the tokens of each sequence, and the sequence of each token."""
    n, lens = s["logp"].numel(), s["seqs"].diff()
    at, inside = _padded(s["seqs"], s["longest"], n)
    if s["mask"] is not None:
        inside = inside & s["mask"][at]
    over = inside.sum(1).clamp_min(1).float() if s["mean"] else torch.ones(len(lens), device="cuda")
    return at, inside, over, torch.arange(len(lens), device="cuda").repeat_interleave(lens, output_size=n)


def _plain_pref(s):
    at, inside, over, seq = _counted(s)
    diff = s["logp"] - s["ref_logp"]
    margins = _BETA * torch.where(inside, diff[at], 0.0).sum(1) / over
    S = margins.numel()
    of, there = _padded(s["groups"], s["largest"], S)
    h, r = margins[of], s["scores"][of]
    ahead = there[:, :, None] & there[:, None, :] & (r[:, :, None] > r[:, None, :])
    d = h[:, :, None] - h[:, None, :]
    e = torch.exp(-d.abs())
    pairs = ahead.sum((1, 2)).clamp_min(1).float()
    loss = torch.where(ahead, (-d).clamp_min(0) + torch.log1p(e) + s["smoothing"] * d, 0.0).sum((1, 2)) / pairs
    slope = torch.where(ahead, s["smoothing"] - torch.where(d >= 0, e, 1.0) / (1.0 + e), 0.0)
    by_h = (slope.sum(2) - slope.sum(1)) / pairs[:, None]
    flat = torch.zeros(S + 1, device="cuda")
    flat[torch.where(there, of, S)] = by_h
    grad = (flat[:S] * _BETA / over)[seq]
    return loss, margins, grad if s["mask"] is None else torch.where(s["mask"], grad, 0.0)


def _plain_adv(s):
    r = s["scores"]
    of, there = _padded(s["groups"], s["largest"], r.numel())
    n = there.sum(1).clamp_min(1).float()
    mean = torch.where(there, r[of], 0.0).sum(1) / n
    off = torch.where(there, r[of] - mean[:, None], 0.0)
    std = torch.sqrt((off * off).sum(1) / n)
    flat = torch.zeros(r.numel() + 1, device="cuda")
    flat[torch.where(there, of, r.numel())] = off / (std + _EPS)[:, None]
    return flat[:-1]


def _plain_policy(s):
    at, inside, over, seq = _counted(s)
    lp, a = s["logp"], s["advantages"][seq]
    ratio, q = torch.exp(lp - s["old_logp"]), s["ref_logp"] - lp
    up = torch.expm1(q)
    loss = _KL * (up - q) - torch.minimum(ratio * a, ratio.clamp(1 - _CLIP_LOW, 1 + _CLIP_HIGH) * a)
    free = torch.where(a >= 0, ratio <= 1 + _CLIP_HIGH, ratio >= 1 - _CLIP_LOW)
    grad = (torch.where(free, -a * ratio, 0.0) - _KL * up) / over[seq]
    if s["mask"] is not None:
        grad = torch.where(s["mask"], grad, 0.0)
    return torch.where(inside, loss[at], 0.0).sum(1) / over, torch.where(inside, (up - q)[at], 0.0).sum(1) / over, grad


_own = {"logp": _own_logp, "grad": _own_grad, "pref": _own_pref, "adv": _own_adv, "policy": _own_policy}
_plain = {"logp": _plain_logp, "grad": _plain_grad, "pref": _plain_pref, "adv": _plain_adv, "policy": _plain_policy}


# ----------------------------------------------------------------------------------------------
# what a pass needs, and its outputs in 64 bits
# ----------------------------------------------------------------------------------------------
def work(case: dict) -> dict:
    if case["call"] in ("logp", "grad"):
        n, size = case["rows"], 4 if case["dtype"] == "f32" else 2
        read = n * (1 - case["ignored"]) * case["vocab"]  # ignored tokens' logits need not be read
        if case["call"] == "logp":
            return {"bytes": read * size + n * (20 + 4 * case["entropy"]), "flops": read * (5 + 2 * case["entropy"])}
        read *= 0.9  # nor those of tokens whose gradients are zero
        if case["entropy"]:
            read /= 0.9
        return {"bytes": (read + n * case["vocab"]) * size + n * (20 + 8 * case["entropy"]), "flops": read * (5 + 3 * case["entropy"])}
    many = (case["few"] + case["many"]) / 2
    S = case["groups"] * many
    if case["call"] == "adv":
        return {"bytes": 8 * S + 8 * case["groups"], "flops": 6 * S}
    lo, hi = case["short"], case["long"]
    tokens = S * (1 - case["empty"]) * ((hi - lo) / math.log(hi / lo) if hi > lo else hi)
    masked = tokens if case["prompt"] else 0
    if case["call"] == "pref":
        pairs = case["groups"] * (many ** 2 + (case["many"] - case["few"]) ** 2 / 12) / 2
        return {"bytes": 12 * tokens + masked + 16 * S + 12 * case["groups"], "flops": 3 * tokens + 16 * pairs}
    return {"bytes": 16 * tokens + masked + 20 * S, "flops": 24 * tokens}


def exact(case: dict, seed: int):
    made = _make(case, seed)
    if case["call"] in ("logp", "grad"):
        return _exact_logits(case, made)
    groups, seqs = _lengths(case, seed)
    host = {k: v.cpu().numpy() for k, v in made.items() if isinstance(v, torch.Tensor)}
    if case["call"] == "adv":
        out = np.zeros(len(host["scores"]))
        for a, b in zip(groups[:-1], groups[1:]):
            r = host["scores"][a:b].astype(np.float64)
            out[a:b] = (r - r.mean()) / (r.std() + _EPS)
        return out
    lp, ref = host["logp"].astype(np.float64), host["ref_logp"].astype(np.float64)
    weight = host["mask"].astype(np.float64) if made["mask"] is not None else np.ones(len(lp))
    lens = np.diff(seqs)

    def total(v):  # the sum over each sequence's tokens that count
        run_ = np.concatenate([[0.0], np.cumsum(v * weight, dtype=np.longdouble)])
        return (run_[seqs[1:]] - run_[seqs[:-1]]).astype(np.float64)

    share = 1.0 / np.maximum(total(np.ones(len(lp))), 1) if case["mean"] else np.ones(len(lens))
    if case["call"] == "pref":
        margins = _BETA * share * total(lp - ref)
        loss, by_h = np.zeros(len(groups) - 1), np.zeros(len(lens))
        for k, (a, b) in enumerate(zip(groups[:-1], groups[1:])):
            i, j = np.nonzero(np.greater.outer(host["scores"][a:b], host["scores"][a:b]))
            if not len(i):
                continue
            d = margins[a + i] - margins[a + j]
            loss[k] = np.mean(np.logaddexp(0.0, -d) + case["smoothing"] * d)
            slope = (case["smoothing"] - 1.0 / (1.0 + np.exp(d))) / len(i)
            by_h[a:b] = np.bincount(i, slope, b - a) - np.bincount(j, slope, b - a)
        return loss, margins, np.repeat(by_h * _BETA * share, lens) * weight
    a = np.repeat(host["advantages"].astype(np.float64), lens)
    ratio = np.exp(lp - host["old_logp"].astype(np.float64))
    kl = np.expm1(ref - lp) - (ref - lp)
    clipped = np.where(a >= 0, ratio > 1 + _CLIP_HIGH, ratio < 1 - _CLIP_LOW)
    edge = np.where(a >= 0, 1 + _CLIP_HIGH, 1 - _CLIP_LOW)
    loss = _KL * kl - a * np.where(clipped, edge, ratio)
    grad = -np.where(clipped, 0.0, a * ratio) - _KL * np.expm1(ref - lp)
    return share * total(loss), share * total(kl), grad * np.repeat(share, lens) * weight


def _exact_logits(case: dict, made: dict):
    n, V = case["rows"], case["vocab"]
    x, t, c = made["logits"], made["targets"], case["scale"]
    live = (t >= 0) & (t < V)
    logp, entropy, stats = (torch.zeros(s, dtype=torch.float64, device="cuda") for s in ((n,), (n,), (n, 2)))
    grads = torch.empty((n, V), dtype=torch.float64, device="cuda") if case["call"] == "grad" else None
    step = max(1, (1 << 28) // V)
    for a in range(0, n, step):
        rows, alive = slice(a, a + step), live[a:a + step]
        y = x[rows].double()
        top = y.amax(1, keepdim=True)
        log_p = torch.log_softmax(c * y, 1)
        p = log_p.exp()
        h = -(p * log_p.masked_fill(p == 0, 0.0)).sum(1)
        at = torch.where(alive, t[rows], 0)[:, None]
        mine = log_p.gather(1, at)[:, 0]
        logp[rows], entropy[rows] = torch.where(alive, mine, 0.0), torch.where(alive, h, 0.0)
        log_sum = torch.logsumexp(c * (y - top), 1, keepdim=True)
        stats[rows] = torch.where(alive[:, None], torch.cat([top, log_sum], 1), 0.0)
        if grads is not None:
            g = made["grad_logp"][rows].double()[:, None] * alive[:, None]
            d = -g * p
            if case["entropy"]:
                k = made["grad_entropy"][rows].double()[:, None] * alive[:, None]
                d -= k * p * (log_p + h[:, None]).masked_fill(p == 0, 0.0)
            grads[rows] = d.scatter_add(1, at, g) * c
    if grads is not None:
        return grads
    return (logp, entropy, stats) if case["entropy"] else (logp, stats)
