"""Performance cases of the operators at the two ends of a training step on scores: the tokens of the answers are
sampled from logits, and the gradients that the losses led to are measured and clipped before the weights take them.

  sample  tokens from temperature, top-k, top-p and min-p, by given random numbers, with their log-probabilities
  norm    the 2-norm of all gradients of a model together
  clip    the norm, and the gradients scaled so that it is at most a limit

Where `own` is false, `run` computes them by elementary torch operations: in 64 bits where a running sum decides on a
token and where the squares of a whole model are added, in 32 bits otherwise.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}

# logits: `rows` tokens to sample of a vocabulary of `vocab`, rows `pad` logits further apart than that. Most tokens'
# logits are noise of `spread`; the likeliest 64 fall off from a peak, which lies `low` to `high` above the mean: far above
# the noise one token takes everything, within it thousands share the probability. `banned`: share of the vocabulary whose
# logits are -inf. `mixed`: every row has parameters of its own, in place of the four. `logp`: log-probabilities are wanted.
_SAMPLE = {"call": "sample", "rows": 1, "vocab": 32_000, "pad": 0, "dtype": "bf16", "spread": 2.0, "low": 13.0, "high": 21.0,
           "banned": 0.0, "scale": 1.0, "top_k": 0, "top_p": 1.0, "min_p": 0.0, "mixed": False, "logp": True}
# gradients of a model of `layers` layers of four width x width and three width x inner matrices and two vectors, and of an
# embedding; `rank`: of adapters of that rank beside the seven matrices instead. `vectors`: the vectors' type. `bucket`: all
# gradients of a type are views into one buffer, one behind the other, beginning at its element `first`. `size`: standard
# deviation of a gradient; `limit`: the norm allowed, as a share of what it is about to be.
_GRADS = {"layers": 2, "width": 512, "inner": 2_048, "vocab": 0, "rank": 0, "dtype": "bf16", "vectors": "bf16", "bucket": False,
          "first": 0, "size": 1e-3, "limit": 0.5}


def _sample(**changes) -> dict:
    return {**_SAMPLE, **changes}


def _grads(call: str, **changes) -> dict:
    return {"call": call, **_GRADS, **changes}


def listed() -> list:
    return [
        # generation for one user: a temperature of 0.8 and the nucleus of 95%
        _sample(name="sample_one", vocab=128_000, scale=1.25, top_p=0.95),
        # a small serving batch in single precision, top-k and the nucleus together, an odd vocabulary
        _sample(name="sample_24_f32_odd", rows=24, vocab=50_001, dtype="f32", top_k=50, top_p=0.9, logp=False),
        # the tokens of 256 answers of 24 tokens from a small table of logits, as the example samples them
        _sample(name="sample_6k_x_136", rows=6_144, vocab=136, dtype="f32", spread=1.0, low=0.0, high=6.0),
        # one step of 256 answers that a policy is trained on: the whole distribution, with log-probabilities
        _sample(name="sample_256_free", rows=256, vocab=128_000),
        # a serving batch whose requests each bring parameters of their own
        _sample(name="sample_512_mixed", rows=512, vocab=131_072, dtype="f16", mixed=True),
        # many prompts' answers of a mid-size vocabulary, part of which a grammar excludes; padded odd rows
        _sample(name="sample_2k_min_p", rows=2_048, vocab=32_001, pad=6, min_p=0.05, banned=0.3),
        # a high temperature and a wide nucleus: thousands of tokens take part
        _sample(name="sample_64_wide", rows=64, vocab=128_000, dtype="f32", low=8.0, high=14.0, scale=0.75, top_p=0.98),
        # the smallest model, in single precision
        _grads("norm", name="norm_small", layers=2, width=128, inner=512, dtype="f32", vectors="f32", size=1e-2),
        # adapters of every matrix of a large model: hundreds of small tensors
        _grads("norm", name="norm_448_adapters", layers=32, width=4_096, inner=8_192, rank=16),
        # a billion weights
        _grads("norm", name="norm_1b", layers=22, width=2_048, inner=4_096, vocab=32_000),
        # a small model whose gradients lie in one buffer, at odd places; too small to be clipped
        _grads("clip", name="clip_small_bucket", layers=6, width=512, inner=2_048, vocab=32_001, dtype="f32", vectors="f32",
               bucket=True, first=1, limit=2.0),
        # two billion weights, vectors in single precision: the largest
        _grads("clip", name="clip_2b_mixed", layers=24, width=2_048, inner=8_192, vocab=128_000, vectors="f32"),
    ]


def _log_int(rng, lo: float, hi: float) -> int:
    return max(int(lo), min(int(hi), int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng) -> dict:
    call = rng.choice(["sample", "sample", "sample", "norm", "clip"])
    if call == "sample":
        vocab = _log_int(rng, 20, 150_000)
        rows = _log_int(rng, 1, min(16_384, (1 << 26) // vocab))
        peak = rng.uniform(4.0, 20.0)
        return _sample(rows=rows, vocab=vocab, pad=rng.choice([0, 0, rng.randint(1, 64)]), dtype=rng.choice(["bf16", "f16", "f32"]),
                       spread=rng.choice([1.0, 2.0, 3.0]), low=round(peak - rng.uniform(0.0, 4.0), 2), high=round(peak, 2),
                       banned=rng.choice([0.0, 0.0, 0.5]), scale=rng.choice([1.0, round(rng.uniform(0.6, 2.0), 3)]),
                       top_k=rng.choice([0, 0, _log_int(rng, 1, 2_000)]), top_p=rng.choice([1.0, round(rng.uniform(0.3, 0.99), 3)]),
                       min_p=rng.choice([0.0, 0.0, round(rng.uniform(0.01, 0.3), 3)]), mixed=rng.random() < 0.25,
                       logp=rng.random() < 0.7)
    width = _log_int(rng, 32, 4_096)
    inner = width * rng.choice([2, 4])
    rank = rng.choice([0, 0, 0, _log_int(rng, 1, 64)])
    layer = 4 * width ** 2 + 3 * width * inner
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    most = 700_000_000 if dtype == "f32" else 1_400_000_000  # weights of the layers
    layers = _log_int(rng, 1, 48 if rank else max(1, min(48, most // layer)))
    return _grads(call, layers=layers, width=width, inner=inner, vocab=0 if rank else _log_int(rng, 10, min(150_000, 2e8 / width)),
                  rank=rank, dtype=dtype, vectors=rng.choice([dtype, "f32"]), bucket=rng.random() < 0.4, first=rng.randint(0, 9),
                  size=rng.choice([1e-4, 1e-3, 1e-2]), limit=rng.choice([0.1, 0.5, 2.0]))


# ----------------------------------------------------------------------------------------------
# inputs
# ----------------------------------------------------------------------------------------------
_EPS = 1e-6


def _random(seed: int) -> torch.Generator:
    return torch.Generator(device="cuda").manual_seed(5 * seed + 1)


def _f32(v: float) -> float:
    """A parameter as the single precision holds it that calls take it in."""
    return float(np.float32(v))


def _make_logits(case: dict, seed: int) -> dict:
    g = _random(seed)
    n, V = case["rows"], case["vocab"]
    wide = torch.empty((n, V + case["pad"]), dtype=_DTYPES[case["dtype"]], device="cuda")
    x = wide[:, :V]
    x.normal_(0.0, case["spread"], generator=g)
    heads = min(64, V)
    peak = case["low"] + (case["high"] - case["low"]) * torch.rand((n, 1), generator=g, device="cuda")
    fall = 1.2 * torch.log(torch.arange(1, heads + 1, device="cuda"))
    head = peak - fall + torch.empty((n, heads), device="cuda").normal_(0.0, 0.5, generator=g)
    # one place in each of `heads` stretches of the vocabulary, the stretches in another order for every row
    stretch = torch.rand((n, heads), generator=g, device="cuda").argsort(1)
    place = ((stretch + torch.rand((n, heads), generator=g, device="cuda")) * (V / heads)).long().clamp_max(V - 1)
    x.scatter_(1, place, head.to(x.dtype))
    if case["banned"]:
        out = torch.rand(V, generator=g, device="cuda") < case["banned"]
        out[0] = False
        x.masked_fill_(out, -math.inf)
    made = {"call": "sample", "logits": x, "uniform": torch.rand(n, generator=g, dtype=torch.float64, device="cuda"), "logp": case["logp"]}
    if not case["mixed"]:
        return made | {"scale": _f32(case["scale"]), "top_k": case["top_k"], "top_p": _f32(case["top_p"]), "min_p": _f32(case["min_p"])}

    def one_of(values, dtype=torch.float32):
        return torch.tensor(values, dtype=dtype, device="cuda")[torch.randint(0, len(values), (n,), generator=g, device="cuda")]

    # greedy requests keep one token; most of the others the nucleus, some with top-k or min-p before it, a few everything
    return made | {"scale": one_of([1.0, 1.0, 1.25, 1 / 0.7]), "top_k": one_of([0, 0, 0, 0, 1, 20, 50, 200], torch.int32),
                   "top_p": one_of([1.0, 0.8, 0.9, 0.95, 0.95]), "min_p": one_of([0.0, 0.0, 0.0, 0.02, 0.1])}


def _shapes(case: dict) -> list:
    """(shape, type) of every gradient, in the model's order."""
    w, i, r, of = case["width"], case["inner"], case["rank"], _DTYPES[case["dtype"]]
    matrices = [(w, w)] * 4 + [(i, w), (i, w), (w, i)]
    if r:
        layer = [(s, of) for a, b in matrices for s in ((a, r), (r, b))]
    else:
        layer = [(m, of) for m in matrices] + [((w,), _DTYPES[case["vectors"]])] * 2
    return ([((case["vocab"], w), of)] if case["vocab"] else []) + layer * case["layers"]


def _numel(shapes: list, dtype=None) -> int:
    return sum(math.prod(s) for s, d in shapes if dtype is None or d == dtype)


def _flat(shapes: list, first: int) -> tuple:
    """One buffer for the tensors of each type, from its element `first` on, and the tensors in order."""
    whole = {d: torch.empty(first + _numel(shapes, d), dtype=d, device="cuda") for d in dict.fromkeys(d for _, d in shapes)}
    at, views = dict.fromkeys(whole, first), []
    for s, d in shapes:
        n = math.prod(s)
        views.append(whole[d][at[d]:at[d] + n].view(s))
        at[d] += n
    return [b[first:] for b in whole.values()], views


def _make_grads(case: dict, seed: int) -> dict:
    g = _random(seed)
    shapes = _shapes(case)
    if case["bucket"]:
        _, grads = _flat(shapes, case["first"])
    else:
        grads = [torch.empty(s, dtype=d, device="cuda") for s, d in shapes]
    sizes = case["size"] * np.exp(np.random.default_rng(seed).normal(0.0, 0.5, len(grads)))
    for t, s in zip(grads, sizes):
        t.normal_(0.0, float(s), generator=g)
    if case["call"] == "norm":
        return {"call": "norm", "grads": grads}
    limit = case["limit"] * math.sqrt(sum(t.numel() * s * s for t, s in zip(grads, sizes)))
    whole, out = _flat(shapes, case["first"] if case["bucket"] else 0)
    return {"call": "clip", "grads": grads, "limit": _f32(limit), "out": out, "whole": whole}


def _make(case: dict, seed: int) -> dict:
    return _make_logits(case, seed) if case["call"] == "sample" else _make_grads(case, seed)


def prepare(case: dict, seed: int) -> dict:
    return _make(case, seed)


# ----------------------------------------------------------------------------------------------
# one pass
# ----------------------------------------------------------------------------------------------
def run(state: dict):
    return (_own if own else _plain)[state["call"]](state)


def _own_sample(s):
    import paper_1212_2287_amd as te

    tokens, logp, log_kept = te.tree_ens_sample(s["logits"], s["uniform"], scale=s["scale"], top_k=s["top_k"], top_p=s["top_p"],
                                                min_p=s["min_p"], want_logp=s["logp"])
    return (tokens, logp, log_kept) if s["logp"] else tokens


def _own_norm(s):
    import paper_1212_2287_amd as te

    return te.tree_ens_grad_norm(s["grads"])


def _own_clip(s):
    import paper_1212_2287_amd as te

    norm = te.tree_ens_grad_norm(s["grads"])
    te.tree_ens_grad_clip(s["grads"], norm, s["limit"], eps=_EPS, out=s["out"])
    return norm, s["whole"]


def _column(v):
    """A parameter in 64 bits, broadcast over the vocabulary where every row has its own."""
    return v.double()[:, None] if isinstance(v, torch.Tensor) else v


def _plain_sample(s):
    x = s["logits"].double()
    scale, top_p, min_p, k = (_column(s[p]) for p in ("scale", "top_p", "min_p", "top_k"))
    z = (x - x.amax(1, keepdim=True)) * scale
    w = torch.exp(z)
    order = torch.sort(x, dim=1, descending=True, stable=True).indices  # equal logits: the lowest index first
    rank = torch.arange(x.shape[1], device="cuda")
    sorted_w = w.gather(1, order)
    inside = sorted_w >= min_p
    limit = torch.where(k > 0, k, x.shape[1]) if isinstance(k, torch.Tensor) else k or x.shape[1]
    inside &= rank < limit
    sorted_w = torch.where(inside, sorted_w, 0.0)
    before = sorted_w.cumsum(1) - sorted_w
    # what comes before a token of the nucleus is less than the nucleus asks for; a top_p of 1 asks for all
    asked = top_p * sorted_w.sum(1, keepdim=True)
    nucleus = (before < asked) | (top_p >= 1.0) if isinstance(top_p, torch.Tensor) else (before < asked) if top_p < 1.0 else inside
    keep = torch.zeros_like(inside).scatter_(1, order, inside & nucleus)
    del order, sorted_w, before, inside, nucleus
    running = torch.where(keep, w, 0.0).cumsum(1)
    tokens = (running <= s["uniform"][:, None] * running[:, -1:]).sum(1)
    if not s["logp"]:
        return tokens
    total = w.sum(1)
    logp = z.gather(1, tokens[:, None])[:, 0] - torch.log(total)
    dropped = torch.where(keep, 0.0, w).sum(1)
    return tokens, logp.float(), torch.log1p(-dropped / total).float()


def _plain_norm(s):
    return torch.stack([t.double().square().sum() for t in s["grads"]]).sum().sqrt().float()


def _plain_clip(s):
    norm = _plain_norm(s)
    factor = torch.clamp_max(s["limit"] / (norm + _EPS), 1.0)
    [o.copy_(t.float() * factor) for t, o in zip(s["grads"], s["out"])]
    return norm, s["whole"]


_own = {"sample": _own_sample, "norm": _own_norm, "clip": _own_clip}
_plain = {"sample": _plain_sample, "norm": _plain_norm, "clip": _plain_clip}


# ----------------------------------------------------------------------------------------------
# what a pass needs, and its outputs in 64 bits
# ----------------------------------------------------------------------------------------------
def work(case: dict) -> dict:
    if case["call"] == "sample":
        n, read = case["rows"], case["rows"] * case["vocab"]
        # the largest logit, and an exponential and a sum of each
        return {"bytes": read * (4 if case["dtype"] == "f32" else 2) + n * (16 + 8 * case["logp"] + 16 * case["mixed"]), "flops": 4 * read}
    shapes = _shapes(case)
    size = sum(math.prod(s) * (4 if d == torch.float32 else 2) for s, d in shapes)
    many = _numel(shapes)
    return {"bytes": size + 4, "flops": 2 * many} if case["call"] == "norm" else {"bytes": 2 * size + 8, "flops": 3 * many}


def exact(case: dict, seed: int):
    made = _make(case, seed)
    return _exact_sample(made) if case["call"] == "sample" else _exact_grads(made)


def _exact_sample(made: dict):
    """By the logit that the last kept token has, and how many of its equals are kept."""
    n, V = made["logits"].shape

    def each(v):
        return v.double()[:, None] if isinstance(v, torch.Tensor) else torch.full((n, 1), float(v), dtype=torch.float64, device="cuda")

    params = [each(made[name]) for name in ("scale", "top_k", "top_p", "min_p", "uniform")]
    tokens, logp, kept = (torch.zeros(n, dtype=t, device="cuda") for t in (torch.int64, torch.float64, torch.float64))
    step = max(1, (1 << 25) // V)
    for a in range(0, n, step):
        rows = slice(a, a + step)
        x = made["logits"][rows].double()
        scale, top_k, top_p, min_p, u = (v[rows] for v in params)
        log_p = torch.log_softmax(scale * x, 1)
        down = torch.sort(log_p, 1, descending=True).values
        many = torch.where(top_k > 0, top_k.clamp_max(V), V)
        many = torch.minimum(many, (down >= down[:, :1] + torch.log(min_p)).sum(1, keepdim=True)).long()
        mass = torch.exp(down).cumsum(1)
        nucleus = torch.searchsorted(mass, top_p * mass.gather(1, many - 1)) + 1
        many = torch.where(top_p < 1, torch.minimum(many, nucleus), many)
        last = torch.sort(x, 1, descending=True).values.gather(1, many - 1)
        spare = many - (x > last).sum(1, keepdim=True)
        level = x == last
        keep = (x > last) | (level & (level.cumsum(1) <= spare))
        prob = torch.exp(log_p)
        mass = torch.where(keep, prob, 0.0).cumsum(1)
        t = torch.searchsorted(mass, u * mass[:, -1:], right=True).clamp_max(V - 1)
        tokens[rows], logp[rows] = t[:, 0], log_p.gather(1, t)[:, 0]
        kept[rows] = torch.log1p(-torch.where(keep, 0.0, prob).sum(1))
    return (tokens, logp, kept) if made["logp"] else tokens


def _exact_grads(made: dict):
    total = sum(float(torch.dot(f, f)) for f in (t.double().reshape(-1) for t in made["grads"]))
    norm = torch.tensor(math.sqrt(total), dtype=torch.float64)
    if made["call"] == "norm":
        return norm
    factor = min(1.0, made["limit"] / (math.sqrt(total) + _EPS))
    types = list(dict.fromkeys(t.dtype for t in made["grads"]))
    return norm, [torch.cat([t.double().reshape(-1) * factor for t in made["grads"] if t.dtype == d]) for d in types]
