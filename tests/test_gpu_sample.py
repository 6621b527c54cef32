"""GPU sampling through the C ABI, against the float64 oracle on the same (already rounded) logits.

Tokens are equal. Weights are off by 2^-39 of themselves and half a unit (2^-45, for fewer than 2^19 tokens) at most, so
what is kept, at least 1, by 2^-39 + 2^-45 V relative; what is not kept is added as it is, in single precision where top_k or
min_p cuts: of u = 2^-24 a weight exp(z) is then off by 3 u |z| (the distance, its product, the exponent) and 4 u (exp2), and
the |z| that count are below 48, so the share D that is not kept by 152 u. logp and the logarithm of the share kept are off by
as much, the latter over the share kept, beside their own rounding, u of them."""
from __future__ import annotations

from fractions import Fraction

import numpy as np
import pytest

from oracle import sampling as O

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def T():
    import paper_1212_2287_amd as T
    T.load_library()
    return T


def _torch_dtype(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[name]


def _logits(dtype, n, V, pad=0, first=0, seed=0, banned=0.0, spread=2.0, peak=9.0):
    """Device logits [n, V] with rows V + pad apart, the first one `first` elements into its allocation, the values
    they stand for, and a random number for each row. Peaks of 0 to `peak` stand out of noise."""
    import torch
    rng = np.random.default_rng([seed, n, V])
    x = rng.normal(0, spread, (n, V))
    for r in range(n):
        at = rng.integers(0, V, min(V, 40))
        x[r, at] += rng.uniform(0, peak) - 0.8 * np.log(np.arange(1, len(at) + 1))
    if banned:
        x[:, rng.random(V) < banned] = -np.inf
        x[:, V // 2] = 1.0
    flat = torch.zeros(first + n * (V + pad), dtype=_torch_dtype(dtype), device="cuda")
    d = flat[first:].view(n, V + pad)[:, :V]
    d.copy_(torch.from_numpy(x))
    return d, d.double().cpu().numpy(), rng.random(n)


def _dev(a, dtype=None):
    import torch
    return torch.from_numpy(np.array(a, dtype=dtype)).cuda()


def _check(got, want, V, what):
    tokens, logp, log_kept = (g.cpu().numpy() for g in got)
    assert np.array_equal(tokens, want[0]), (what, np.nonzero(tokens != want[0])[0][:5], tokens[:5], want[0][:5])
    off = 2.0 ** -39 + 2.0 ** -45 * max(V, 1) * max(1.0, V / 2 ** 18)
    quick = 152 * U * -np.expm1(want[2])
    for name, a, b, e in (("logp", logp, want[1], off + quick + U * np.abs(want[1])),
                          ("log_kept", log_kept, want[2], (2 * off + quick) / np.exp(want[2]) + U * np.abs(want[2]))):
        fine = np.isfinite(b)
        assert np.array_equal(a[~fine], b[~fine], equal_nan=True), (what, name)
        err = np.abs(a[fine].astype(np.float64) - b[fine]) - e[fine]
        assert (err <= 0).all(), (what, name, float(err.max()))
    assert not (log_kept > 0).any()


def _f32(v):
    return float(np.float32(v))


SHAPES = [
    # tokens, vocabulary, padding of a row, elements before the first row
    (1, 1, 0, 0), (3, 2, 0, 0), (5, 7, 1, 1), (9, 63, 0, 0), (4, 64, 0, 0), (300, 65, 0, 3), (17, 255, 2, 0), (8, 257, 0, 1),
    (30, 1000, 0, 0), (33, 1023, 0, 0), (6, 2047, 2, 5), (5, 2048, 0, 0), (3, 2049, 7, 0), (5, 4095, 0, 0), (4, 4097, 1, 0),
    (4, 8193, 8, 0), (2, 20_001, 0, 0), (5, 32_000, 0, 0), (2, 65_537, 0, 1), (2, 131_072, 0, 0), (6, 50_001, 0, 0),
]
PARAMS = [
    dict(), dict(scale=0.7), dict(top_k=1), dict(top_k=50), dict(top_k=700), dict(top_p=0.9), dict(top_p=0.3, scale=1.6),
    dict(min_p=0.05), dict(top_k=40, top_p=0.8, min_p=0.01), dict(top_k=5_000, top_p=0.97), dict(min_p=1.0), dict(top_p=1e-6),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,V,pad,first", SHAPES)
def test_against_the_oracle(T, dtype, n, V, pad, first):
    what = f"{dtype} {n} x {V} + {pad} from {first}"
    print("[sample]", what, flush=True)
    for k, params in enumerate(PARAMS):
        if n * V > 100_000 and k % 3 != (n + V) % 3:
            continue
        params = {p: v if p == "top_k" else _f32(v) for p, v in params.items()}
        d, x, u = _logits(dtype, n, V, pad, first, seed=k, banned=0.4 if k % 2 else 0.0, peak=(14.0, 3.0)[k % 5 == 0])
        got = T.tree_ens_sample(d, _dev(u), **params)
        _check(got, O.sample(x, u, **params), V, (what, params))
        tokens, none, also = T.tree_ens_sample(d, _dev(u), want_logp=False, **params)
        assert none is None and also is None and (tokens == got[0]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V", [1, 2, 5, 300, 3000, 5000, 40_000])
def test_rows_of_special_values(T, dtype, V):
    import torch
    lowest = torch.finfo(_torch_dtype(dtype)).min
    n = 12
    x = np.random.default_rng(V).normal(0, 2, (n, V))
    x[0] = -np.inf                     # nothing can be sampled
    x[1] = -np.inf
    x[1, V - 1] = 2.0                  # one token
    x[2] = lowest                      # masked by the lowest value, all alike
    x[3] = lowest
    x[3, V - 1] = 0.5
    x[4, V // 2] = np.nan
    x[5, V // 2] = np.inf
    x[6] = 0.0                         # equals by index, whatever the sign of their zero
    x[6, ::2] = -0.0
    x[7] = -lowest                     # the largest
    x[8] = np.where(np.arange(V) % 3, 1.0, 2.0)
    x[9, V // 2] = -np.nan
    x[10] = -np.inf
    x[10, V // 3:V // 3 + 2] = [-lowest, lowest][:len(x[10, V // 3:V // 3 + 2])]
    x[11, 0] = -lowest
    d = torch.from_numpy(x).to(_torch_dtype(dtype)).cuda()
    x = d.double().cpu().numpy()
    for k, params in enumerate(({}, dict(top_k=2), dict(top_p=0.5), dict(min_p=0.5), dict(top_k=max(V - 1, 1), top_p=0.75, min_p=0.25))):
        for u in (np.random.default_rng(k).random(n), np.zeros(n), np.full(n, 1 - 2.0 ** -53)):
            _check(T.tree_ens_sample(d, _dev(u), **params), O.sample(x, u, **params), V, (dtype, V, params, u[0]))


@pytest.mark.parametrize("V", [1000, 6000, 70_000])
@pytest.mark.parametrize("levels", [1, 2, 7])
def test_many_equal_logits(T, V, levels):
    """Borders of top-k and top-p inside runs of equals, far longer than any list of candidates: the first by index stay."""
    rng = np.random.default_rng([V, levels])
    n = 16
    x = rng.integers(0, levels, (n, V)) * 0.75
    d, u = _dev(x, np.float32), rng.random(n)
    top_p = rng.uniform(0.01, 0.99, n).astype(np.float32)
    top_k = rng.integers(1, V + 1, n).astype(np.int32)
    for dtype in ("f32", "bf16", "f16"):
        for params in (dict(top_p=top_p), dict(top_k=top_k), dict(top_k=top_k, top_p=top_p), dict(min_p=0.3, top_p=top_p)):
            given = {k: _dev(v) if isinstance(v, np.ndarray) else _f32(v) for k, v in params.items()}
            params = {k: v if isinstance(v, np.ndarray) else _f32(v) for k, v in params.items()}
            _check(T.tree_ens_sample(d.to(_torch_dtype(dtype)), _dev(u), **given), O.sample(x, u, **params), V, (V, levels, dtype, list(params)))


@pytest.mark.parametrize("n", [3, 260])
@pytest.mark.parametrize("V,spread", [(20_000, 0.001), (70_001, 0.02), (70_001, 0.5), (300_000, 0.2)])
def test_many_near_equals(T, n, V, spread):
    """Thousands of logits that differ little around the last kept one, in rows that workgroups share and in more of them."""
    import torch
    x = torch.empty(n, V, device="cuda").normal_(0, spread, generator=torch.Generator("cuda").manual_seed(V))
    u = torch.rand(n, dtype=torch.float64, device="cuda", generator=torch.Generator("cuda").manual_seed(n))
    some = [0, n // 2, n - 1]
    for more in (dict(top_p=_f32(0.4)), dict(top_k=V // 2), dict(top_k=V // 3, top_p=_f32(0.6)), dict(top_k=V // 3, min_p=_f32(0.9)),
                 dict(top_p=_f32(0.5), min_p=_f32(0.5))):
        got = T.tree_ens_sample(x, u, **more)
        want = O.sample(x[some].double().cpu().numpy(), u[some].cpu().numpy(), **more)
        _check([g[some] for g in got], want, V, more)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [2_049, 2_055, 4_097, 6_143, 6_145, 50_001, 65_537, 65_541])
def test_candidates_at_the_ends_of_the_row(T, dtype, V):
    """The likeliest tokens are the row's first and last ones, which share loads and segments with what lies beyond it."""
    rng = np.random.default_rng(V)
    n = 12
    x = rng.normal(0, 1, (n, V))
    x[:, :9] += 9.0
    x[:, -9:] += 9.0
    x[6:, -3:] = 11.5  # equals
    d = _dev(np.concatenate([x, np.full((n, 5), 30.0)], 1)).to(_torch_dtype(dtype))[:, :V]  # larger ones beyond
    x, u = d.double().cpu().numpy(), np.concatenate([rng.random(n - 2), [0.0, 1 - 2.0 ** -53]])
    for params in (dict(), dict(top_k=1), dict(top_k=17), dict(top_k=60), dict(top_p=0.9), dict(min_p=_f32(0.02)),
                   dict(top_k=V - 3, top_p=_f32(0.95)), dict(top_p=_f32(0.999)), dict(top_k=V - 1)):
        params = {k: v if k == "top_k" else _f32(v) for k, v in params.items()}
        _check(T.tree_ens_sample(d, _dev(u), **params), O.sample(x, u, **params), V, (V, dtype, params))


@pytest.mark.parametrize("dtype,n,V", [("bf16", 40, 300), ("f32", 24, 5_000), ("f16", 16, 60_001)])
def test_parameters_of_each_row(T, dtype, n, V):
    d, x, u = _logits(dtype, n, V, seed=4)
    rng = np.random.default_rng(V)
    scale = rng.uniform(0.5, 2.0, n).astype(np.float32)
    top_k = np.where(rng.random(n) < 0.5, 0, rng.integers(1, V, n)).astype(np.int32)
    top_p = np.where(rng.random(n) < 0.4, 1.0, rng.random(n)).astype(np.float32)
    min_p = np.where(rng.random(n) < 0.5, 0.0, rng.uniform(0, 0.2, n)).astype(np.float32)
    got = T.tree_ens_sample(d, _dev(u), scale=_dev(scale), top_k=_dev(top_k), top_p=_dev(top_p), min_p=_dev(min_p))
    _check(got, O.sample(x, u, scale, top_k, top_p, min_p), V, "rows' own")
    _check(T.tree_ens_sample(d, _dev(u), scale=1.25, top_p=_dev(top_p)), O.sample(x, u, 1.25, 0, top_p), V, "some of them")
    # beyond their ranges: (given, what it counts as)
    for name, kind, given, counts in (("top_k", np.int32, [-3, 0, V, V + 9, 2**31 - 1], [0, 0, 0, 0, 0]),
                                      ("top_p", np.float32, [-1.0, 0.0, 1.5, np.inf, np.nan], [1e-9, 1e-9, 1, 1, 1]),
                                      ("min_p", np.float32, [-1.0, 0.0, 1.5, np.inf, np.nan], [0, 0, 1, 1, 0])):
        got = T.tree_ens_sample(d[:5], _dev(u[:5]), **{name: _dev(given, kind)})
        _check(got, O.sample(x[:5], u[:5], **{name: counts}), V, (name, "beyond its range"))
    wrong = _dev([1.0, 0.0, -1.0, np.inf, np.nan], np.float32)
    tokens, logp, log_kept = (t.cpu().numpy() for t in T.tree_ens_sample(d[:5], _dev(u[:5]), scale=wrong))
    assert tokens[0] >= 0 and (tokens[1:] == -1).all() and np.isnan(logp[1:]).all() and np.isnan(log_kept[1:]).all()


def test_random_numbers_at_the_borders(T):
    """Weights that are exact: a running sum that the random number equals is not past it. Others count as the nearest
    in [0, 1), NaN as 0."""
    for V in (4, 4096, 8192):
        u = np.array([0.0, 0.25, 0.5, 0.75, 0.25 - 2.0 ** -53, 0.75 - 2.0 ** -53, 1 - 2.0 ** -53])
        d = _dev(np.zeros((len(u), V)), np.float32)
        assert T.tree_ens_sample(d, _dev(u))[0].tolist() == [int(f * V) for f in u]
        assert T.tree_ens_sample(d, _dev(u), top_k=4)[0].tolist() == [0, 1, 2, 3, 0, 2, 3]
        beyond = np.array([-0.5, 1.0, 2.0, np.inf, -np.inf, np.nan, -0.0])
        assert T.tree_ens_sample(d, _dev(beyond))[0].tolist() == [0, V - 1, V - 1, V - 1, 0, 0, 0]


@pytest.mark.parametrize("V", [50, 6_000])
def test_even_random_numbers_give_the_distribution(T, V):
    """n even random numbers hit a token n p times, give or take one."""
    import torch
    n = 4_000
    d, x, _ = _logits("f32", 1, V, seed=2)
    u = (np.arange(n) + 0.5) / n
    tokens, _, _ = T.tree_ens_sample(d.repeat(n, 1), _dev(u), scale=1.5, top_k=30, top_p=0.875)
    order, w = O.kept_tokens(x[0], 1.5, 30, 0.875)
    p = np.zeros(V)
    p[order] = w[order] / w[order].sum()
    assert np.abs(np.bincount(tokens.cpu().numpy(), minlength=V) - n * p).max() <= 1 + 1e-6
    assert isinstance(tokens, torch.Tensor) and tokens.dtype == torch.int64


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [60, 900, 2_500, 70_000])
def test_shares_not_kept_however_small(T, dtype, V):
    """Rows of which almost nothing is dropped, down to 1e-13 of the probability, and then nothing at all: the logarithm of the
    share kept is right in proportion. Single precision: 152 u of it; what is left of a sum whose tokens are taken out of it again
    counts as nothing up to 2^-44, which a row of 35 parts may do in each."""
    n = 12
    rng = np.random.default_rng(V)
    x = rng.normal(0, 1, (n, V))
    x[np.arange(n), rng.integers(0, V, n)] = np.linspace(12, 32, n)
    x[:, rng.permutation(V)[:20]] += 6.0
    d = _dev(x).to(_torch_dtype(dtype))
    x, u = d.double().cpu().numpy(), rng.random(n)
    for params in (dict(top_k=1), dict(top_k=15), dict(top_k=V - V // 8), dict(min_p=_f32(1e-3)), dict(top_p=0.5), dict(top_k=V // 2, top_p=0.75)):
        want = O.sample(x, u, **params)
        tokens, logp, log_kept = (t.double().cpu().numpy() for t in T.tree_ens_sample(d, _dev(u), **params))
        assert np.array_equal(tokens, want[0])
        assert (np.abs(log_kept - want[2]) <= 153 * U * np.abs(want[2]) + 40 * 2.0 ** -44).all(), (params, log_kept, want[2])
        assert (np.abs(logp - want[1]) <= 153 * U * -np.expm1(want[2]) + U * np.abs(want[1]) + 2.0 ** -39 + 2.0 ** -45 * V).all()
    # masked beyond the first: nothing has a weight that is not kept
    d[:, 10:] = -float("inf")
    for params in (dict(top_k=10), dict(top_k=11), dict(min_p=_f32(1e-30)), dict(top_k=min(V, 500), min_p=_f32(1e-30))):
        assert not T.tree_ens_sample(d, _dev(u), **params)[2].any(), params


@pytest.mark.parametrize("V", [700, 9_000])
def test_scales_of_any_size(T, V):
    rng = np.random.default_rng(V)
    x = rng.normal(0, 3, (6, V)).astype(np.float32)
    u = rng.random(6)
    for scale in (1e-30, 1e-6, 0.01, 30.0, 1e6, 3e38):
        for params in ({}, dict(min_p=0.1), dict(top_p=0.5), dict(top_k=V // 2)):
            params = {k: v if k == "top_k" else _f32(v) for k, v in params.items()}
            _check(T.tree_ens_sample(_dev(x), _dev(u), scale=_f32(scale), **params), O.sample(x, u, _f32(scale), **params), V, (scale, params))


@pytest.mark.parametrize("V", [524_287, 524_288, 3_000_001])
def test_the_largest_vocabularies(T, V):
    """Units grow so that the sum stays in its 63 bits; equal weights of a power of two are exact all the same."""
    import torch
    d = torch.zeros(3, V, dtype=torch.bfloat16, device="cuda")
    d[1, ::2] = -1.0
    u = np.array([0.5, 0.25, 0.999])
    x = d.double().cpu().numpy()
    tokens, logp, _ = (t.cpu().numpy() for t in T.tree_ens_sample(d, _dev(u)))
    w = np.exp(x)
    for r in range(3):
        c = np.cumsum(w[r])
        assert abs(tokens[r] - np.searchsorted(c, u[r] * c[-1], side="right")) <= (0 if r != 1 else 1)
        assert abs(logp[r] - (x[r, tokens[r]] - np.log(c[-1]))) <= 2 * U * abs(logp[r])
    kept = T.tree_ens_sample(d[1:2].repeat(3, 1), _dev(u), top_k=_dev([1, 1000, V // 2], np.int32))
    order = 1 + 2 * np.arange(V // 2)
    # the product of the random number as it is, which a double's would round up to a whole number at 1,500,000 tokens
    assert kept[0].tolist() == [order[0], order[250], order[int(Fraction(u[2]) * (V // 2))]]


def test_rows_do_not_depend_on_their_batch(T):
    for dtype, n, V in (("bf16", 600, 5_000), ("f32", 70, 33_001), ("f16", 300, 300)):
        d, _, u = _logits(dtype, n, V, seed=6)
        u = _dev(u)
        whole = T.tree_ens_sample(d, u, top_p=0.9)
        for r in (0, 1, n // 2, n - 1):
            for a, b in zip(whole, T.tree_ens_sample(d[r:r + 1], u[r:r + 1], top_p=0.9)):
                assert (a[r:r + 1] == b).all(), (dtype, r)


def test_another_stream_and_equal_bits(T):
    import torch
    d, _, u = _logits("bf16", 37, 30_011)
    u = _dev(u)
    side = torch.cuda.Stream()
    first = T.tree_ens_sample(d, u, top_p=0.8)
    side.wait_stream(torch.cuda.current_stream())
    again = T.tree_ens_sample(d, u, top_p=0.8, stream=side)
    raw = T.tree_ens_sample(d, u, top_p=0.8, stream=side.cuda_stream)
    side.synchronize()
    for a, b, c in zip(first, again, raw):
        assert torch.equal(a, b) and torch.equal(a, c)


def test_two_calls_at_once(T):
    """Calls on two streams with workspaces of their own."""
    import torch
    d, _, u = _logits("f32", 64, 20_000, seed=1)
    e, _, v = _logits("f32", 64, 20_000, seed=2)
    u, v = _dev(u), _dev(v)
    want = [T.tree_ens_sample(d, u, top_p=0.9), T.tree_ens_sample(e, v, top_k=30)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        got = [T.tree_ens_sample(d, u, top_p=0.9), T.tree_ens_sample(e, v, top_k=30, stream=side)]
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert all(torch.equal(a, b) for a, b in zip(g, w))


def test_offsets_past_32_bits(T):
    """Rows whose logits lie beyond 2^31 elements (and 2^32 bytes) of the first."""
    import torch
    n, stride = 5, 600_000_000
    flat = torch.empty((n - 1) * stride + 9_000, dtype=torch.bfloat16, device="cuda")
    for V in (1000, 9_000):
        d = flat.as_strided((n, V), (stride, 1))
        x = torch.from_numpy(np.random.default_rng(0).normal(0, 2, (n, V))).to(torch.bfloat16)
        d.copy_(x)
        u = np.random.default_rng(1).random(n)
        _check(T.tree_ens_sample(d, _dev(u), top_p=_f32(0.9)), O.sample(x.double().numpy(), u, top_p=_f32(0.9)), V, "far rows")


@pytest.mark.parametrize("V,more", [(5, dict(top_p=0.9)), (2_055, dict(top_p=0.9)), (2_055, dict(top_p=0.9, spread=0.1)), (2_055, {})],
                         ids=["short", "listed", "wide", "all"])
def test_more_rows_than_workgroups(T, V, more):
    """More rows than a launch has workgroups: the first and the last ones are as in calls of their own."""
    import torch
    n, some = (1 << 20) + 77, 60
    x = torch.empty(n, V, dtype=torch.bfloat16, device="cuda").normal_(0, more.get("spread", 3.0), generator=torch.Generator("cuda").manual_seed(1))
    u = torch.rand(n, dtype=torch.float64, device="cuda", generator=torch.Generator("cuda").manual_seed(2))
    top_p = _f32(more.get("top_p", 1.0))
    got = T.tree_ens_sample(x, u, top_p=top_p)
    assert ((got[0] >= 0) & (got[0] < V)).all() and torch.isfinite(got[1]).all() and (got[2] <= 0).all()
    for rows in (slice(0, some), slice(n - some, n)):
        part = [g[rows] for g in got]
        assert all(torch.equal(a, b) for a, b in zip(part, T.tree_ens_sample(x[rows], u[rows], top_p=top_p)))
        _check(part, O.sample(x[rows].double().cpu().numpy(), u[rows].cpu().numpy(), top_p=top_p), V, "rows in turn")


@pytest.mark.parametrize("n,V", [(3, 60_001), (40, 500)])
def test_captured_into_a_graph(T, n, V):
    import torch
    d, _, _ = _logits("f32", n, V)
    u = torch.rand(n, dtype=torch.float64, device="cuda")
    out = [torch.empty(n, dtype=torch.int64, device="cuda"), torch.empty(n, device="cuda"), torch.empty(n, device="cuda")]
    top_p = torch.full((n,), 0.9, device="cuda")

    def step():
        T.tree_ens_sample(d, u, top_p=top_p, tokens=out[0], logp=out[1], log_kept=out[2])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        g = torch.Generator().manual_seed(k)
        d.copy_(torch.randn(d.shape, generator=g) * 3)
        u.copy_(torch.rand(n, generator=g, dtype=torch.float64))
        top_p.copy_(torch.rand(n, generator=g))
        step()
        want = [o.clone() for o in out]
        for o in out:
            o.fill_(-7)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b), k


def test_logp_is_that_of_token_logp(T):
    """Both give log softmax(scale * row)[token]; token_logp's error is that of single-precision sums of the row."""
    import torch
    for dtype, n, V in (("bf16", 200, 32_000), ("f32", 50, 700)):
        d, _, u = _logits(dtype, n, V, seed=9)
        tokens, logp, _ = T.tree_ens_sample(d, _dev(u), scale=1.25, top_k=20)
        want, _, stats = T.tree_ens_token_logp(d, tokens, scale=1.25)
        z = 4 * (1 + want.abs() + stats[:, 1].abs()) + V / 256 + 72
        assert torch.all((logp - want).abs() <= U * (z + want.abs()))
    d[0] = -float("inf")
    tokens, _, _ = T.tree_ens_sample(d, _dev(u))
    assert tokens[0] == -1 and T.tree_ens_token_logp(d, tokens)[0][0] == 0  # a row that does not count


def test_only_rows_of_the_call_are_written(T):
    import torch
    d, _, u = _logits("bf16", 5, 6_001)
    wide = [torch.full((9,), -7, dtype=t, device="cuda") for t in (torch.int64, torch.float32, torch.float32)]
    T.tree_ens_sample(d, _dev(u), top_p=0.9, tokens=wide[0][2:7], logp=wide[1][2:7], log_kept=wide[2][2:7])
    for w in wide:
        assert (w[:2] == -7).all() and (w[7:] == -7).all() and (w[2:7] != -7).all()


def test_argument_errors(T):
    import torch
    d, _, u = _logits("f32", 3, 8)
    u = _dev(u)
    for bad in (u.float(), u[:2], u.repeat(2)[::2]):
        with pytest.raises(TypeError, match="uniform"):
            T.tree_ens_sample(d, bad)
    with pytest.raises(TypeError, match="contiguous rows"):
        T.tree_ens_sample(d.t(), _dev(np.zeros(8)))
    with pytest.raises(TypeError, match="logits"):
        T.tree_ens_sample(d.double(), u)
    with pytest.raises(TypeError, match="top_k"):
        T.tree_ens_sample(d, u, top_k=torch.ones(3, device="cuda"))
    with pytest.raises(TypeError, match="scale"):
        T.tree_ens_sample(d, u, scale=torch.ones(2, device="cuda"))
    with pytest.raises(TypeError, match="top_p"):
        T.tree_ens_sample(d, u, top_p=torch.ones(3))
    with pytest.raises(TypeError, match="tokens"):
        T.tree_ens_sample(d, u, tokens=torch.empty(3, dtype=torch.int32, device="cuda"))
    with pytest.raises(TypeError, match="logp"):
        T.tree_ens_sample(d, u, logp=torch.empty(2, device="cuda"))
    for bad in (dict(scale=0.0), dict(top_k=-1), dict(top_p=0.0), dict(min_p=2.0)):
        with pytest.raises(T.TreeEnsError) as ei:
            T.tree_ens_sample(d, u, **bad)
        assert ei.value.code == T.TREE_ENS_E_ARG
    with pytest.raises(T.TreeEnsError):
        T.tree_ens_sample(d[:1].expand(3, 8), u)  # rows that share their logits
    tokens, logp, log_kept = T.tree_ens_sample(torch.empty(0, 8, device="cuda"), u[:0])
    assert tokens.shape == logp.shape == log_kept.shape == (0,)
    assert (T.tree_ens_sample(d, u, top_k=2**40)[0] == T.tree_ens_sample(d, u)[0]).all()


LARGE = [dict(top_k=1), dict(top_k=40), dict(min_p=0.05), dict(top_k=40, top_p=0.75), dict(top_p=0.5)]


@pytest.mark.parametrize("V", [3_000, 9_001, 40_001])
@pytest.mark.parametrize("scale", [7e7, 1e10, 1e12, 1e30])
def test_masked_logits_under_large_scales(T, scale, V):
    """Logits some 1 / scale apart, beside others (and ends of rows) whose distance is no float once it is scaled."""
    import torch
    scale, rng, n = _f32(scale), np.random.default_rng(V), 7
    x = rng.normal(0, 2, (n, V)) / scale
    x[1:3, rng.random(V) < 0.3] = -np.inf
    x[3:5, rng.random(V) < 0.3] = torch.finfo(torch.float32).min
    x[5] = -1.0
    x[5, [0, V - 1]] = 0.0, -0.7 / scale
    x[6] = -np.inf
    x[6, [1, V // 2, V - 2]] = 0.0, -0.7 / scale, -1.5 / scale
    x, u = x.astype(np.float32), rng.random(n)
    for params in [*LARGE, dict(top_k=V // 2)]:
        params = {k: v if k == "top_k" else _f32(v) for k, v in params.items()}
        _check(T.tree_ens_sample(_dev(x), _dev(u), scale=scale, **params), O.sample(x, u, scale, **params), V, (scale, params))


@pytest.mark.parametrize("V", [700, 3_000, 9_001])
@pytest.mark.parametrize("scale", [1e38, 2.4e38, 3.4e38])
def test_scales_up_to_the_largest(T, scale, V):
    """Scales that the exponential's base makes too large for a float, on logits that are subnormal."""
    scale, rng, n = _f32(scale), np.random.default_rng(V), 4
    x = rng.normal(0, 2, (n, V)) / scale
    x[1, rng.random(V) < 0.3] = -np.inf
    x[2:, V // 2:] = -1.0
    x, u = x.astype(np.float32), rng.random(n)
    for params in [*LARGE, dict(top_k=V // 2)]:
        params = {k: v if k == "top_k" else _f32(v) for k, v in params.items()}
        _check(T.tree_ens_sample(_dev(x), _dev(u), scale=scale, **params), O.sample(x, u, scale, **params), V, (scale, params))


def _check_shares(got, want, V, quick, what):
    """log_kept in proportion to the share D that is not kept, however small: the weights' and sums' errors twice (in D and in
    the total), 152 u where single precision adds what is dropped, what of 1 - D is lost where it is small, the rounding to float,
    half its smallest step at least."""
    assert np.array_equal(got[0].cpu().numpy(), want[0]), what
    D = -np.expm1(want[2])
    off = 2.0 ** -39 + 2.0 ** -45 * V * max(1.0, V / 2 ** 18)
    tol = D * (2 * off + (152 * U if quick else 0.0) + 2.0 ** -50 / (1 - D)) + U * np.abs(want[2]) + 2.0 ** -150
    err = np.abs(got[2].double().cpu().numpy() - want[2])
    assert (err <= tol).all(), (what, got[2].tolist(), want[2].tolist(), (err / tol).max())


@pytest.mark.parametrize("mask", ["-inf", "lowest"])
@pytest.mark.parametrize("V,ahead", [(2, 1), (60, 3), (900, 20), (524_300, 2)])
def test_far_tokens_not_kept(T, V, ahead, mask):
    """What is dropped is e^-40 to e^-100 of the rest, and the other tokens are masked: in short rows and in rows too long for a digest."""
    rng, n = np.random.default_rng(V), 13 if V < 1_000 else 4
    x = np.full((n, V), -np.inf if mask == "-inf" else np.finfo(np.float32).min, np.float32)
    for r, z in enumerate(np.linspace(40, 100, n)):
        order = rng.permutation(V)
        x[r, order[:ahead]] = rng.normal(0, 1, ahead)
        x[r, order[0]] = 2.5  # the largest, with which a nucleus of half begins
        far = order[ahead:ahead + max(1, V // 3)]
        x[r, far] = 2.5 - z - rng.random(len(far))
    u = rng.random(n)
    for params in (dict(top_k=ahead), dict(top_k=ahead + V // 6), dict(min_p=_f32(1e-7))):
        _check_shares(T.tree_ens_sample(_dev(x), _dev(u), **params), O.sample(x, u, **params), V, False, (V, mask, params))


@pytest.mark.parametrize("n", [13, 300])
@pytest.mark.parametrize("V", [5_000, 40_001])
@pytest.mark.parametrize("first,last", [(40, 66), (65, 100)])
def test_far_tokens_of_wide_rows(T, first, last, V, n):
    """Rows of which more is kept than a list holds, and further tokens e^-`first` to e^-`last` of those, of which some are kept
    as well: in rows that workgroups share and in more of them."""
    rng = np.random.default_rng(V)
    x = np.full((n, V), -np.inf, np.float32)
    for r, z in enumerate(np.linspace(first, last, n)):
        order = rng.permutation(V)
        x[r, order[:1_000]] = rng.normal(0, 1, 1_000)
        x[r, order[0]] = 2.5
        x[r, order[1_000:3_000]] = 2.5 - z - rng.random(2_000)
    u, some = rng.random(n), np.arange(0, n, max(1, n // 13))
    for params in (dict(top_k=1_000), dict(top_k=1_700), dict(top_k=3_000), dict(top_k=3_001), dict(top_k=1_700, min_p=_f32(1e-30)),
                   dict(min_p=_f32(1e-7)), dict(top_p=_f32(0.95)), dict(top_k=1_700, top_p=_f32(0.95))):
        got = [g[_dev(some)] for g in T.tree_ens_sample(_dev(x), _dev(u), **params)]
        _check_shares(got, O.sample(x[some], u[some], **params), V, False, (first, V, n, params))


@pytest.mark.parametrize("V,ahead,there", [(2_500, 1, 3), (2_500, 40, 60), (2_500, 90, 300), (40_001, 5, 400), (5_000, 600, 700), (140_000, 600, 3_000)])
def test_far_tokens_of_a_list(T, V, ahead, there):
    """The same of tokens that a list of candidates holds beside the kept ones, the first `ahead` of `there`, or a bin of more
    candidates than a list holds beside the last ones kept, 20 further ones."""
    rng, n = np.random.default_rng(V + there), 9
    x = np.full((n, V), -np.inf, np.float32)
    for r, z in enumerate(np.linspace(30, 62, n)):
        order = rng.permutation(V)[:there]
        x[r, order] = -z - np.arange(there) * (3.0 / there)
        x[r, order[:ahead]] = 0.0
    u = rng.random(n)
    params = dict(min_p=_f32(1e-30), top_p=_f32(1 - 0.5 / ahead)) if there <= 512 else dict(top_k=ahead + 20)
    _check_shares(T.tree_ens_sample(_dev(x), _dev(u), **params), O.sample(x, u, **params), V, True, (V, there))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [2_049, 4_096, 40_001, 140_000])
def test_far_tokens_beside_a_list(T, dtype, V):
    """The same of tokens that share a part of the row with the kept ones and are in no list: some rows have them in every part,
    some in one, and some none at all."""
    rng, n = np.random.default_rng(V), 16
    x = np.full((n, V), -np.inf)
    for r, z in enumerate(np.linspace(12, 100, n)):
        at = rng.integers(0, V)
        if r % 4 == 1:
            x[r] = -z - rng.random(V)
        elif r % 4 == 2:
            x[r, max(0, at - 300):at + 300] = -z
        elif r % 4 == 3:
            x[r, (at + 1) % V] = -z
        x[r, at] = 0.0
        if r % 3 == 0:
            x[r, rng.integers(0, V, 20)] = -rng.random(20)
    d = _dev(x).to(_torch_dtype(dtype))
    x, u = d.double().cpu().numpy(), rng.random(n)
    for params in (dict(top_k=1), dict(top_k=15), dict(min_p=_f32(1e-3)), dict(top_p=0.25), dict(top_p=_f32(0.99))):
        got, want = T.tree_ens_sample(d, _dev(u), **params), O.sample(x, u, **params)
        _check_shares(got, want, V, True, (dtype, V, params))
        assert not got[2].cpu().numpy()[want[2] == 0.0].any()


def test_numbers_of_tokens_to_keep_that_are_no_int32(T):
    d, _, u = _logits("f32", 3, 8)
    u = _dev(u)
    for top_k in (-2**31, -2**31 - 1, -2**32 + 5, -2**40):
        with pytest.raises(T.TreeEnsError) as ei:
            T.tree_ens_sample(d, u, top_k=top_k)
        assert ei.value.code == T.TREE_ENS_E_ARG
    assert (T.tree_ens_sample(d, u, top_k=2**32 + 1)[0] == T.tree_ens_sample(d, u)[0]).all()


@pytest.mark.parametrize("V,spread", [(128_000, 1.0), (140_001, 0.01)])
def test_rows_do_not_depend_on_how_many_workgroups_share_them(T, V, spread):
    """Wide nuclei: a row alone goes to many workgroups, the rows of a batch to fewer, those of a large one to one each. Bits are equal."""
    import torch
    x = torch.empty(300, V, device="cuda").normal_(0, spread, generator=torch.Generator("cuda").manual_seed(V))
    u = torch.rand(300, dtype=torch.float64, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    for params in (dict(top_p=0.97), dict(top_k=V // 3), dict(top_k=V // 2, top_p=0.9), dict(min_p=0.2)):
        alone = [T.tree_ens_sample(x[r:r + 1], u[r:r + 1], **params) for r in (0, 3)]
        for n in (2, 9, 40, 64, 130, 200, 256, 257, 300):
            got = T.tree_ens_sample(x[:n], u[:n], **params)
            for r, want in zip((0, 3), alone):
                assert r >= n or all(torch.equal(g[r:r + 1], w) for g, w in zip(got, want)), (V, params, n, r)
