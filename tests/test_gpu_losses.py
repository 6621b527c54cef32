"""GPU preference loss, group advantages and policy loss through the C ABI, against the float64 oracle.

Tolerances, with u = 2^-24: differences of log-probabilities are rounded once, exp and log1p are off by at most
8u, sums are held in double and rounded once. A margin is off by u (sum of its terms + itself); a pair's loss and
slope by the two margins' errors (both have slope <= 1) plus 16u."""
from __future__ import annotations

import numpy as np
import pytest

from oracle import losses as O

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def T():
    import paper_1212_2287_amd as T
    T.load_library()
    return T


def _dev(a):
    import torch
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _close(got, want, tol, what):
    got = got.double().cpu().numpy()
    assert got.shape == np.shape(want), what
    fine = np.isfinite(want)
    assert np.array_equal(got[~fine], want[~fine], equal_nan=True), what
    err = np.abs(got - want)[fine] / (np.broadcast_to(tol, np.shape(want))[fine] + 1e-37)
    assert (err <= 1).all(), (what, float(err.max()), int(err.argmax()))


# lengths of the sequences
LENGTHS = {
    "none": [], "one": [1], "empty": [0, 0, 0], "pair": [3, 2], "edges": [0, 1, 2, 63, 64, 65, 0, 127, 128, 129, 255, 256, 257, 0],
    "short": list(np.random.default_rng(1).integers(0, 9, 700)), "mixed": list(np.random.default_rng(2).integers(1, 700, 300)),
    "tile": [2047, 1, 2048, 2049, 4096, 3, 6145, 0, 5], "long": [100_003, 7, 0, 40_000], "single": [262_147],
    "skewed": [1] * 500 + [90_001] + [2] * 500, "many": list(np.random.default_rng(3).integers(0, 40, 20_000)),
    "ordinary": list(np.random.default_rng(4).integers(1, 1200, 2_000)),
}


def _tokens(name, seed=0, masked=True):
    rng = np.random.default_rng([seed, len(name)])
    lens = np.array(LENGTHS[name], np.int64)
    seqs = np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)
    n = int(seqs[-1])
    lp = -rng.exponential(size=n).astype(np.float32)
    ref = (lp + rng.normal(0, 0.3, n)).astype(np.float32)
    mask = None
    if masked:
        mask = rng.random(n) < 0.7
        for s in rng.integers(0, max(len(lens), 1), len(lens) // 10):  # sequences of which nothing counts
            mask[seqs[s]:seqs[s + 1]] = False
    return rng, seqs, lp, ref, mask


def _groups(rng, n_seqs, sizes):
    """Group offsets of the given sizes in turn, as many as there are sequences."""
    ends = []
    at = 0
    while at < n_seqs:
        at = min(n_seqs, at + int(sizes[len(ends) % len(sizes)]))
        ends.append(at)
    return np.concatenate([[0], ends]).astype(np.int64)


def _check_preference(T, seqs, lp, ref, mask, scores, groups, beta, smoothing, grad_scale, mean, what):
    flags = T.TREE_ENS_SEQ_MEAN if mean else 0
    args = (_dev(lp), _dev(seqs), _dev(scores), _dev(groups))
    more = dict(ref_logp=_dev(ref), mask=_dev(mask), beta=beta, smoothing=smoothing, grad_scale=grad_scale, flags=flags)
    loss, h, grad = T.tree_ens_preference_loss(*args, **more)
    beta, smoothing, grad_scale = (float(np.float32(v)) for v in (beta, smoothing, grad_scale))
    want = O.preference_loss(lp, seqs, scores, groups, ref, mask, beta, smoothing, grad_scale, mean)
    size = O.margins(np.abs(lp if ref is None else lp.astype(np.float64) - ref), seqs, None, mask, abs(beta), mean)[0]
    tol_h = 2 * U * (size + np.abs(want[1]))
    _close(h, want[1], tol_h, what + " margins")
    tol_loss, tol_grad, w = np.zeros(len(groups) - 1), np.zeros(len(seqs) - 1), np.abs(O.margins(lp, seqs, ref, mask, beta, mean)[1])
    for g, (a, b) in enumerate(zip(groups[:-1], groups[1:])):
        s = scores[a:b]
        pairs = max(int((s[:, None] > s[None, :]).sum()), 1)
        worst, span = 2 * tol_h[a:b].max(initial=0), np.ptp(want[1][a:b]) if b > a else 0.0
        each = worst + U * span + 16 * U
        tol_loss[g] = each + 8 * U * want[0][g] + 2 * U * abs(smoothing) * span
        met = (s[:, None] > s[None, :]).sum(1) + (s[:, None] < s[None, :]).sum(1)
        tol_grad[a:b] = abs(grad_scale) * w[a:b] * met / pairs * (each + 8 * U)
    _close(loss, want[0], tol_loss, what + " loss")
    per_token = np.repeat(tol_grad, np.diff(seqs)) + 4 * U * np.abs(want[2])
    _close(grad, want[2], per_token, what + " gradient")
    only = T.tree_ens_preference_loss(*args, **more, want_grad=False)
    assert only[2] is None and bool((only[0] == loss).all()) and bool((only[1] == h).all())
    again = T.tree_ens_preference_loss(*args, **more)
    assert all(bool((x == y).all()) for x, y in zip(again, (loss, h, grad)))


@pytest.mark.parametrize("sizes", [[2], [1, 5, 0, 17, 64], [130, 7], [1500]])
@pytest.mark.parametrize("name", [k for k in LENGTHS if k not in ("none",)])
def test_preference_loss(T, name, sizes):
    print("[preference]", name, sizes, flush=True)
    for k, (mean, masked, smoothing) in enumerate([(False, True, 0.0), (True, False, 0.1), (True, True, 0.3)]):
        rng, seqs, lp, ref, mask = _tokens(name, k, masked)
        n_seqs = len(seqs) - 1
        groups = _groups(rng, n_seqs, sizes)
        scores = np.round(rng.normal(size=n_seqs) * 4).astype(np.float32) / 4  # equal scores among them
        scores[rng.random(n_seqs) < 0.05] = np.nan
        _check_preference(T, seqs, lp, ref if k else None, mask, scores, groups, 0.1 if k else 0.01, smoothing, 0.25, mean,
                          f"{name} {sizes} {k}")


def test_preference_loss_of_far_margins(T):
    """Margins hundreds apart: losses of thousands one way, of next to nothing the other."""
    lp = np.array([-1.0, -900.0, -2.0, -30.0, -0.5, -20.0], np.float32)
    seqs = np.arange(7)
    scores = np.array([1, 0, 0, 1, 2, 1], np.float32)
    for beta in (1.0, 4.0):
        _check_preference(T, seqs, lp, None, None, scores, np.array([0, 2, 4, 6]), beta, 0.0, 1.0, False, "far")


def test_masked_tokens_may_hold_anything(T):
    rng, seqs, lp, ref, mask = _tokens("mixed")
    old = (lp - rng.normal(0, 0.05, len(lp))).astype(np.float32)
    bad = [np.nan, np.inf, -np.inf]
    dirty = [a.copy() for a in (lp, ref, old)]
    for k, a in enumerate(dirty):
        a[~mask] = np.resize(bad[k:] + bad[:k], int((~mask).sum()))
    groups, n_seqs = _groups(rng, len(seqs) - 1, [9]), len(seqs) - 1
    scores = rng.normal(size=n_seqs).astype(np.float32)
    for mean in (0, T.TREE_ENS_SEQ_MEAN):
        a, b = (T.tree_ens_preference_loss(_dev(x), _dev(seqs), _dev(scores), _dev(groups), ref_logp=_dev(y), mask=_dev(mask),
                                           flags=mean) for x, y in ((lp, ref), dirty[:2]))
        assert all(bool((x == y).all()) for x, y in zip(a, b))
        a, b = (T.tree_ens_policy_loss(_dev(x), _dev(z), _dev(scores), _dev(seqs), ref_logp=_dev(y), mask=_dev(mask),
                                       kl_coef=0.1, flags=mean) for x, y, z in ((lp, ref, old), dirty))
        assert all(bool((x == y).all()) for x, y in zip(a, b))


def _check_policy(T, seqs, lp, old, ref, mask, adv, low, high, kl_coef, grad_scale, mean, what):
    args = (_dev(lp), _dev(old), _dev(adv), _dev(seqs))
    more = dict(ref_logp=_dev(ref), mask=_dev(mask), clip_low=low, clip_high=high, kl_coef=kl_coef, grad_scale=grad_scale,
                flags=T.TREE_ENS_SEQ_MEAN if mean else 0)
    loss, kl, grad = T.tree_ens_policy_loss(*args, **more)
    low, high = 1 - float(np.float32(1) - np.float32(low)), float(np.float32(1) + np.float32(high)) - 1
    kl_coef, grad_scale = float(np.float32(kl_coef)), float(np.float32(grad_scale))
    want = O.policy_loss(lp, old, adv, seqs, ref, mask, low, high, kl_coef, grad_scale, mean)
    n = len(lp)
    use = np.ones(n, bool) if mask is None else mask
    d = np.zeros(n) if old is None else lp.astype(np.float64) - old
    q = np.zeros(n) if ref is None else ref.astype(np.float64) - lp
    A = np.abs(np.repeat(adv, np.diff(seqs))).astype(np.float64)
    e_ratio = U * (8 + 2 * np.abs(d)) * np.exp(d)
    e_kl = 16 * U * (np.expm1(q) - q) + U * np.abs(q * np.expm1(q)) + np.where(np.abs(q) >= 0.5, 8 * U * (np.exp(q) + np.abs(q)), 0)
    e_up = e_kl + 4 * U * (np.abs(q) + np.abs(np.expm1(q)))

    def total(v):
        c = np.concatenate([[0.0], np.cumsum(np.where(use, v, 0.0))])
        return c[seqs[1:]] - c[seqs[:-1]]
    share = 1.0 / np.maximum(total(np.ones(n)), 1) if mean else np.ones(len(seqs) - 1)
    gain = A * np.exp(np.abs(d))
    _close(loss, want[0], share * total(A * e_ratio + 4 * U * gain + abs(kl_coef) * e_kl) + 4 * U * np.abs(want[0]), what + " loss")
    if ref is None:
        assert kl is None
    else:
        _close(kl, want[1], share * total(e_kl) + 4 * U * np.abs(want[1]), what + " kl")
    per = abs(grad_scale) * np.repeat(share, np.diff(seqs)) * (A * e_ratio + abs(kl_coef) * e_up + 4 * U * (gain + np.abs(kl_coef * np.expm1(q))))
    _close(grad, want[2], per, what + " gradient")
    only = T.tree_ens_policy_loss(*args, **more, want_grad=False)
    assert only[2] is None and bool((only[0] == loss).all())
    again = T.tree_ens_policy_loss(*args, **more)
    assert bool((again[0] == loss).all()) and bool((again[2] == grad).all())


@pytest.mark.parametrize("name", list(LENGTHS))
def test_policy_loss(T, name):
    print("[policy]", name, flush=True)
    for k, (mean, masked) in enumerate([(False, False), (True, True), (True, False), (False, True)]):
        rng, seqs, lp, ref, mask = _tokens(name, k, masked)
        n = len(lp)
        r = rng.normal(0, 0.2, n)
        for edge in (np.log(0.8), np.log(1.25)):  # the gradient jumps at a clip's edge
            r = np.where(np.abs(r - edge) < 1e-3, edge + 2e-3, r)
        old = (lp - r).astype(np.float32)
        ref[rng.random(n) < 0.02] += 1.0
        adv = rng.normal(size=len(seqs) - 1).astype(np.float32)
        adv[rng.random(len(adv)) < 0.1] = 0.0
        _check_policy(T, seqs, lp, old, ref if k != 2 else None, mask, adv, 0.2, 0.25, 0.05 if k != 2 else 0.0, 0.5, mean,
                      f"{name} {k}")


def test_policy_loss_on_the_edge_and_far_off(T):
    """Ratios exactly 1 with a clip of nothing count as inside; ratios that overflow are clipped for a positive
    advantage and for an advantage of 0; on-policy tokens have ratio 1."""
    lp = np.array([-1.0, -1.0, 0.0, 0.0, -200.0, -0.5], np.float32)
    old = np.array([-1.0, -1.0, -200.0, -200.0, 0.0, -0.5], np.float32)
    seqs = np.arange(7)
    adv = np.array([2.0, -2.0, 1.0, 0.0, -3.0, 0.0], np.float32)
    _check_policy(T, seqs, lp, old, None, None, adv, 0.0, 0.0, 0.0, 1.0, False, "edge")
    _check_policy(T, seqs, lp, None, lp - np.float32(0.125), None, adv, 0.2, 0.2, 0.5, 1.0, True, "on policy")
    loss, _, grad = T.tree_ens_policy_loss(_dev(lp[2:3]), _dev(old[2:3]), _dev(np.array([-1.0], np.float32)), _dev(np.array([0, 1])))
    assert float(loss) == np.inf and float(grad) == np.inf
    loss, _, grad = T.tree_ens_policy_loss(_dev(np.array([np.nan], np.float32)), _dev(old[:1]), _dev(adv[:1]), _dev(np.array([0, 1])))
    assert np.isnan(float(loss)) and np.isnan(float(grad))


@pytest.mark.parametrize("sizes", [[1], [2], [16], [0, 1, 63, 64, 65, 200], [1025, 3], [5000], [70_000]])
def test_group_advantage(T, sizes):
    rng = np.random.default_rng(len(sizes))
    n = max(3000, 2 * max(sizes))
    groups = _groups(rng, n, sizes)
    scores = (5 + 0.1 * rng.normal(size=n)).astype(np.float32)
    scores[groups[1]:groups[2]] = 2.5  # a group without spread
    for flags in (0, T.TREE_ENS_CENTER_ONLY):
        got = T.tree_ens_group_advantage(_dev(scores), _dev(groups), eps=1e-3, flags=flags)
        want = O.group_advantage(scores, groups, float(np.float32(1e-3)), bool(flags))
        # the sums are double: the result is rounded once (twice if the mean is)
        _close(got, want, 4 * U * np.abs(want) + 1e-12, f"{sizes} {flags}")
    x = _dev(scores)
    T.tree_ens_group_advantage(x, _dev(groups), eps=1e-3, flags=T.TREE_ENS_CENTER_ONLY, advantages=x)
    assert bool((x == got).all())


def test_group_advantage_of_special_scores(T):
    scores = np.array([1.0, np.nan, 2.0, 1.0, np.inf, 3.0, 3.0, 7.0], np.float32)
    got = T.tree_ens_group_advantage(_dev(scores), _dev(np.array([0, 3, 5, 7]))).cpu().numpy()
    assert np.isnan(got[:5]).all() and got[5:].tolist() == [0.0, 0.0, 0.0]


def test_ill_formed_offsets_stay_inside(T):
    """Offsets beyond the tokens are clamped; tokens and sequences outside every segment get zeros."""
    rng, _, lp, ref, _ = _tokens("mixed")
    lp, ref = lp[:1000], ref[:1000]
    seqs = np.array([100, 200, 450, 450, 2000, 2000])
    groups = np.array([1, 3, 9])
    scores = np.arange(5).astype(np.float32)
    loss, h, grad = T.tree_ens_preference_loss(_dev(lp), _dev(seqs), _dev(scores), _dev(groups), ref_logp=_dev(ref))
    want = O.preference_loss(lp, seqs, scores, groups, ref, beta=float(np.float32(0.1)))
    _close(loss, want[0], 1e-5, "loss")
    _close(h, want[1], 1e-4, "margins")
    _close(grad, want[2], 1e-6, "gradient")
    assert not bool(grad[:200].any())
    adv = T.tree_ens_group_advantage(_dev(scores), _dev(groups))
    assert float(adv[0]) == 0.0 and bool((adv[1:3] != 0).all())
    pol = T.tree_ens_policy_loss(_dev(lp), None, _dev(scores), _dev(seqs))
    _close(pol[2], O.policy_loss(lp, None, scores, seqs)[2], 1e-6, "policy gradient")
    # offsets that decrease: whatever comes out, nothing outside is touched
    odd = np.array([500, 20, 900, -7, 10**15, 3])
    guard = _dev(np.full(1000 + 64, 7.0, np.float32))
    T.tree_ens_policy_loss(_dev(lp), None, _dev(scores), _dev(odd), grad_logp=guard[32:1032])
    T.tree_ens_preference_loss(_dev(lp), _dev(odd), _dev(scores), _dev(np.array([3, 0, 10**15, -2])), grad_logp=guard[32:1032])
    assert bool((guard[:32] == 7).all()) and bool((guard[1032:] == 7).all())


def test_nothing_to_learn_from(T):
    import torch
    none, zero = torch.empty(0, device="cuda"), _dev(np.zeros(1, np.int64))
    loss, h, grad = T.tree_ens_preference_loss(none, zero, none, zero)
    assert loss.numel() == h.numel() == grad.numel() == 0
    tokens = torch.ones(300, device="cuda")
    out = torch.full((300,), 5.0, device="cuda")
    T.tree_ens_preference_loss(tokens, zero, none, zero, grad_logp=out)
    assert not bool(out.any())
    out.fill_(5.0)
    T.tree_ens_policy_loss(tokens, None, none, zero, grad_logp=out)
    assert not bool(out.any())
    assert T.tree_ens_group_advantage(none, zero).numel() == 0
    out.fill_(5.0)
    T.tree_ens_group_advantage(tokens, zero, advantages=out)
    assert not bool(out.any())
    out.fill_(5.0)  # sequences, but no group: margins, and a gradient of zeros
    _, h, _ = T.tree_ens_preference_loss(tokens, _dev(np.array([0, 100, 300])), _dev(np.ones(2, np.float32)), zero, beta=0.5, grad_logp=out)
    assert h.tolist() == [50.0, 100.0] and not bool(out.any())


def test_gradients_by_differences(T):
    """The GPU's gradients against differences of the GPU's own losses summed in float64: a step of 0.05 along a
    random direction through 200 tokens has an error of order step^2."""
    import torch
    rng = np.random.default_rng(11)
    seqs, groups = np.arange(0, 201, 10), np.array([0, 8, 20])
    lp, ref = -rng.exponential(size=200), -rng.exponential(size=200)
    scores = rng.normal(size=20).astype(np.float32)
    u = rng.normal(size=200)

    def pref(e, **kw):
        return T.tree_ens_preference_loss(_dev((lp + e * u).astype(np.float32)), _dev(seqs), _dev(scores), _dev(groups),
                                          ref_logp=_dev(ref.astype(np.float32)), smoothing=0.05, flags=T.TREE_ENS_SEQ_MEAN, **kw)
    slope = (pref(0.05)[0].double().sum() - pref(-0.05)[0].double().sum()) / 0.1
    assert abs(float(slope) - float((pref(0.0)[2].double().cpu() * torch.from_numpy(u)).sum())) < 1e-4

    def policy(e):
        return T.tree_ens_policy_loss(_dev((lp + e * u).astype(np.float32)), _dev((lp - 0.05 * u).astype(np.float32)), _dev(scores),
                                      _dev(seqs), ref_logp=_dev(ref.astype(np.float32)), clip_low=1.0, clip_high=9.0, kl_coef=0.2)
    slope = (policy(0.01)[0].double().sum() - policy(-0.01)[0].double().sum()) / 0.02
    got = float((policy(0.0)[2].double().cpu() * torch.from_numpy(u)).sum())
    assert abs(float(slope) - got) < 1e-3 * (1 + abs(got))


def test_another_stream_and_graph(T):
    import torch
    rng, seqs, lp, ref, mask = _tokens("ordinary")
    n_seqs = len(seqs) - 1
    groups = _groups(rng, n_seqs, [30])
    a = [_dev(x) for x in (lp, seqs, rng.normal(size=n_seqs).astype(np.float32), groups, ref, mask)]
    out = [torch.empty(len(groups) - 1, device="cuda"), torch.empty(n_seqs, device="cuda"), torch.empty(len(lp), device="cuda"),
           torch.empty(n_seqs, device="cuda"), torch.empty(n_seqs, device="cuda"), torch.empty(len(lp), device="cuda")]

    def step(stream=None):
        T.tree_ens_preference_loss(a[0], a[1], a[2], a[3], ref_logp=a[4], mask=a[5], flags=T.TREE_ENS_SEQ_MEAN, loss=out[0],
                                   margins=out[1], grad_logp=out[2], stream=stream)
        adv = T.tree_ens_group_advantage(a[2], a[3], stream=stream)
        T.tree_ens_policy_loss(a[0], a[4], adv, a[1], ref_logp=a[4], mask=a[5], kl_coef=0.1, flags=T.TREE_ENS_SEQ_MEAN,
                               loss=out[3], kl=out[4], grad_logp=out[5], stream=stream)
        return adv
    step()
    want = [o.clone() for o in out]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(out, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        adv = step()
    for k in range(3):
        a[0].copy_(torch.from_numpy(-np.random.default_rng(k).exponential(size=len(lp))).float())
        step()
        want = [o.clone() for o in out]
        for o in out:
            o.fill_(-7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(out, want)), k
    assert adv.numel() == n_seqs


def test_argument_errors(T):
    import torch
    lp, seqs = torch.zeros(8, device="cuda"), _dev(np.array([0, 3, 8]))
    scores, groups = torch.zeros(2, device="cuda"), _dev(np.array([0, 2]))
    with pytest.raises(TypeError, match="scores"):
        T.tree_ens_preference_loss(lp, seqs, scores[:1], groups)
    with pytest.raises(TypeError, match="seq_offsets"):
        T.tree_ens_preference_loss(lp, seqs.int(), scores, groups)
    with pytest.raises(TypeError, match="mask"):
        T.tree_ens_preference_loss(lp, seqs, scores, groups, mask=lp)
    with pytest.raises(TypeError, match="ref_logp"):
        T.tree_ens_preference_loss(lp, seqs, scores, groups, ref_logp=lp[:4])
    with pytest.raises(TypeError, match="logp"):
        T.tree_ens_preference_loss(lp.double(), seqs, scores, groups)
    with pytest.raises(T.TreeEnsError) as ei:
        T.tree_ens_preference_loss(lp, seqs, scores, groups, smoothing=1.0)
    assert ei.value.code == T.TREE_ENS_E_ARG
    with pytest.raises(TypeError, match="advantages"):
        T.tree_ens_policy_loss(lp, None, scores[:1].expand(2), seqs)
    with pytest.raises(T.TreeEnsError):
        T.tree_ens_policy_loss(lp, None, scores, seqs, kl_coef=0.1)
    with pytest.raises(T.TreeEnsError):
        T.tree_ens_group_advantage(scores, groups, eps=0.0)


@pytest.mark.parametrize("groups,sizes,length", [
    (300, [2], (1, 60)), (700, [1, 2, 6], (0, 30)),            # one kernel
    (6_000, [2], (1, 40)), (900, [8, 1, 40, 3], (0, 20)),      # few candidates a group, larger ones among them
    (120, [40, 90, 3], (0, 60)), (1, [64], (1, 9)),            # a workgroup a group
    (9, [700, 300, 511, 512, 513], (0, 12)), (2, [1030], (1, 5)), (1, [2100], (1, 3)), (4, [97], (0, 4_000)),  # parts of one
    (30, [600, 2, 31, 1], (0, 9)),                             # groups that differ widely
])
def test_every_way_to_meet_the_pairs(T, groups, sizes, length):
    rng = np.random.default_rng([groups, len(sizes)])
    goff = np.concatenate([[0], np.cumsum(np.resize(sizes, groups))]).astype(np.int64)
    n_seqs = int(goff[-1])
    seqs = np.concatenate([[0], np.cumsum(rng.integers(length[0], length[1] + 1, n_seqs))]).astype(np.int64)
    n = int(seqs[-1])
    lp = -rng.exponential(size=n).astype(np.float32)
    ref = (lp + rng.normal(0, 0.3, n)).astype(np.float32)
    mask = rng.random(n) < 0.8
    scores = (np.round(rng.normal(size=n_seqs) * 8) / 8).astype(np.float32)
    scores[rng.random(n_seqs) < 0.01] = np.nan
    for smoothing, mean in ((0.0, False), (0.2, True)):
        _check_preference(T, seqs, lp, ref, mask, scores, goff, 0.2, smoothing, 1.0, mean, f"{groups} of {sizes}")


@pytest.mark.parametrize("repeat", [1, 40_000])
def test_impossible_tokens_without_old_or_reference_policy(T, repeat):
    """log-probabilities of -inf: without the old policy's the ratio is 1, without a reference the KL term is 0."""
    lp = np.tile(np.array([-1.0, -np.inf, -2.0, -0.5], np.float32), repeat)
    old = np.tile(np.array([-1.0, -3.0, -2.5, -0.5], np.float32), repeat)
    seqs = np.arange(0, 4 * repeat + 1, 2)
    adv = np.resize(np.array([1.0, -1.0], np.float32), 2 * repeat)
    for o in (None, old):
        loss, kl, grad = T.tree_ens_policy_loss(_dev(lp), _dev(o), _dev(adv), _dev(seqs), clip_low=0.5, clip_high=0.5)
        with np.errstate(invalid="ignore"):
            want = O.policy_loss(lp, o, adv, seqs, clip_low=0.5, clip_high=0.5)
        _close(loss, want[0], 1e-5, "loss")
        _close(grad, want[2], 1e-5, "gradient")
        assert kl is None


@pytest.mark.parametrize("seqs_,length", [(3, (0, 50)), (2_000, (40, 60)), (30_000, (0, 5)), (50, (3_000, 20_000)), (3, (200_000, 300_000))])
def test_every_way_to_take_the_tokens_of_a_policy_loss(T, seqs_, length):
    rng = np.random.default_rng(seqs_)
    seqs = np.concatenate([[0], np.cumsum(rng.integers(length[0], length[1] + 1, seqs_))]).astype(np.int64)
    n = int(seqs[-1])
    lp = -rng.exponential(size=n).astype(np.float32)
    r = rng.normal(0, 0.2, n)
    for edge in (np.log(0.8), np.log(1.25)):
        r = np.where(np.abs(r - edge) < 1e-3, edge + 2e-3, r)
    old, ref = (lp - r).astype(np.float32), (lp + rng.normal(0, 0.3, n)).astype(np.float32)
    adv, mask = rng.normal(size=seqs_).astype(np.float32), rng.random(n) < 0.6
    for mean in (False, True):
        for m in (None, mask):
            _check_policy(T, seqs, lp, old, ref, m, adv, 0.2, 0.25, 0.05, 0.5, mean, f"{seqs_} {length} {mean}")


@pytest.mark.parametrize("repeat", [1, 50_000])
def test_tokens_that_one_model_excludes(T, repeat):
    """Infinite log ratios to the reference: the KL term is infinite, its gradient that of exp(q) - 1; without a
    coefficient it is reported and leaves the loss alone."""
    lp = np.tile(np.array([-1.0, -2.0, -np.inf, -0.5], np.float32), repeat)
    ref = np.tile(np.array([-1.5, -np.inf, -3.0, -0.5], np.float32), repeat)
    seqs, adv = np.arange(4 * repeat + 1), np.resize(np.array([1.0, -2.0, 0.5], np.float32), 4 * repeat)
    for kl_coef in (0.0, 0.25):
        got = T.tree_ens_policy_loss(_dev(lp), None, _dev(adv), _dev(seqs), ref_logp=_dev(ref), kl_coef=kl_coef)
        want = O.policy_loss(lp, None, adv, seqs, ref, kl_coef=kl_coef)
        for a, b, what in zip(got, want, ("loss", "kl", "gradient")):
            _close(a, b, 1e-6 * (1 + np.abs(np.where(np.isfinite(b), b, 0.0))), f"{what} {kl_coef}")


@pytest.mark.parametrize("n,length", [(2, 3), (40, 3), (200, 2), (700, 1), (2_500, 1)])
def test_preference_loss_of_close_margins_far_from_zero(T, n, length):
    """Margins about 1,000 that differ by hundredths: the loss goes by their differences, which the rounding of the
    margins themselves (2^-24 of 1,000) limits and nothing else."""
    rng = np.random.default_rng(n)
    lp = (-1000.0 / length + 0.01 * rng.normal(size=n * length)).astype(np.float32)
    seqs, groups = np.arange(0, n * length + 1, length), np.array([0, n])
    scores = rng.normal(size=n).astype(np.float32)
    loss, h, grad = T.tree_ens_preference_loss(_dev(lp), _dev(seqs), _dev(scores), _dev(groups), beta=1.0)
    # the pairs of the margins as they were rounded
    m = h.double().cpu().numpy()
    want = O.preference_loss(m, np.arange(n + 1), scores, groups, beta=1.0)
    _close(h, O.margins(lp, seqs, beta=1.0)[0], 2 * U * 1100, "margins")
    _close(loss, want[0], 40 * U, "loss")
    pairs = n * (n - 1) / 2
    per = (n - 1) / pairs * 40 * U
    _close(grad, np.repeat(want[2], length), per + 4 * U * np.abs(np.repeat(want[2], length)), "gradient")


# groups and their sizes, for each of the ways pairs are met
WAYS = {"one kernel": (40, [8]), "few": (1_100, [8, 2]), "a workgroup": (30, [40]), "its windows": (60, [20] * 29 + [700]),
        "parts": (5, [130]), "windows of parts": (1, [2_500])}


def _margins_alone(way, seed, spread):
    """Sequences of one token, so that a margin is its log-probability: (log-probabilities, sequence and group offsets,
    scores)."""
    count, sizes = WAYS[way]
    groups = np.concatenate([[0], np.cumsum(np.resize(sizes, count))]).astype(np.int64)
    rng = np.random.default_rng([seed, count])
    n = int(groups[-1])
    return (spread * rng.normal(size=n)).astype(np.float32), np.arange(n + 1), groups, rng.normal(size=n).astype(np.float32)


def _per_pair(scores, groups):
    """How many pairs a candidate is in, over the group's number of pairs."""
    out = np.zeros(len(scores))
    for a, b in zip(groups[:-1], groups[1:]):
        ahead = scores[a:b, None] > scores[None, a:b]
        out[a:b] = (ahead.sum(0) + ahead.sum(1)) / max(int(ahead.sum()), 1)
    return out


@pytest.mark.parametrize("first", [0.0, -50.0, -5_000.0, -50_000.0, 1e30])
@pytest.mark.parametrize("way", list(WAYS))
def test_one_far_candidate_leaves_the_other_pairs_exact(T, way, first):
    """Margins of spread 0.3 and one far off, in front of its group: each pair goes by the difference of its own two
    margins, of one rounding. A pair's slope is off by 32 u, and a chain of 128 floats adds 64 u to each at most."""
    lp, seqs, groups, scores = _margins_alone(way, 1, 0.3)
    lp[groups[:-1]] = first
    for smoothing in (0.0, 0.125):
        loss, h, grad = T.tree_ens_preference_loss(_dev(lp), _dev(seqs), _dev(scores), _dev(groups), beta=1.0, smoothing=smoothing)
        assert np.array_equal(h.cpu().numpy(), lp)
        with np.errstate(over="ignore"):
            want = O.preference_loss(lp, seqs, scores, groups, beta=1.0, smoothing=smoothing)
        _close(loss, want[0], 100 * U * (1 + want[0]), f"{way} loss")
        _close(grad, want[2], 100 * U * _per_pair(scores, groups) + 4 * U * np.abs(want[2]), f"{way} gradient")


@pytest.mark.parametrize("smoothing", [0.0, 0.125])
@pytest.mark.parametrize("way", list(WAYS))
def test_margins_of_impossible_answers(T, way, smoothing):
    """An answer that the model excludes has margin -inf: a pair that wants it ahead costs infinitely much, one that wants it
    behind nothing without smoothing and infinitely much with it; the slopes are those of the sigmoid's ends."""
    lp, seqs, groups, scores = _margins_alone(way, 2, 1.0)
    some = groups[:-1][::2]  # in every other group: its first answer, as good as its neighbours or the worst of all
    lp[some] = -np.inf
    scores[some[1::2]] = -9.0
    loss, h, grad = T.tree_ens_preference_loss(_dev(lp), _dev(seqs), _dev(scores), _dev(groups), beta=1.0, smoothing=smoothing)
    assert np.array_equal(h.cpu().numpy(), lp)
    want, slope = np.zeros(len(groups) - 1), np.zeros(len(lp))
    for g, (a, b) in enumerate(zip(groups[:-1], groups[1:])):
        i, j = np.nonzero(scores[a:b, None] > scores[None, a:b])
        d = lp[a + i].astype(np.float64) - lp[a + j]
        each = (1 - smoothing) * np.logaddexp(0, -d)
        if smoothing:
            each += smoothing * np.logaddexp(0, d)
        want[g] = each.mean()
        with np.errstate(over="ignore"):
            dl = (smoothing - 1 / (1 + np.exp(d))) / len(i)
        np.add.at(slope, a + i, dl)
        np.add.at(slope, a + j, -dl)
    _close(loss, want, 100 * U * (1 + np.where(np.isfinite(want), want, 0.0)), "loss")
    _close(grad, slope, 100 * U * _per_pair(scores, groups) + 4 * U * np.abs(slope), "gradient")


@pytest.mark.parametrize("count,sizes", [(3_000, [2] * 99 + [9, 64, 65]), (2_200, [2] * 1_099 + [100]), (5_000, [2] * 1_666 + [700]),
                                         (5_000, [2] * 4_998 + [3_000, 1])])
def test_a_large_group_among_small_ones(T, count, sizes):
    rng = np.random.default_rng([count, len(sizes)])
    groups = np.concatenate([[0], np.cumsum(np.resize(sizes, count))]).astype(np.int64)
    n_seqs = int(groups[-1])
    seqs = np.concatenate([[0], np.cumsum(rng.integers(0, 8, n_seqs))]).astype(np.int64)
    n = int(seqs[-1])
    lp, ref = -rng.exponential(size=n).astype(np.float32), -rng.exponential(size=n).astype(np.float32)
    scores = (np.round(rng.normal(size=n_seqs) * 8) / 8).astype(np.float32)
    for smoothing, mean in ((0.0, False), (0.2, True)):
        _check_preference(T, seqs, lp, ref, rng.random(n) < 0.8, scores, groups, 0.2, smoothing, 1.0, mean, f"{count} of {sizes}")


def test_time_of_a_large_group_among_small_ones(T):
    """16 million ordered pairs of one group, met by 256 threads: 63,000 in a row for each, of some 35 instructions that
    take four cycles: 4 ms and what they wait for. Eight threads would take 110 ms and more."""
    import torch
    groups = _dev(np.concatenate([np.arange(0, 10_000, 2), [14_000]]))
    lp, seqs = -torch.rand(14_000, device="cuda"), torch.arange(14_001, device="cuda")
    scores = torch.randn(14_000, device="cuda")
    times = []
    for _ in range(3):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        T.tree_ens_preference_loss(lp, seqs, scores, groups)
        b.record()
        b.synchronize()
        times.append(a.elapsed_time(b))
    assert min(times) < 40, times


@pytest.mark.parametrize("count,sizes,lengths", [(300, [2], [7] * 399 + [100_003]), (60, [3, 8, 1], [400] * 9 + [4_096, 4_097, 0]),
                                                 (1, [8], [0, 1, 5_000, 1, 2, 3, 1, 2]), (200, [1, 2, 0], [3] * 150 + [60_000] * 2)])
def test_long_answers_among_short_ones_in_small_batches(T, count, sizes, lengths):
    rng = np.random.default_rng([count, len(lengths)])
    groups = np.concatenate([[0], np.cumsum(np.resize(sizes, count))]).astype(np.int64)
    n_seqs = int(groups[-1])
    seqs = np.concatenate([[0], np.cumsum(np.resize(lengths, n_seqs))]).astype(np.int64)
    assert seqs[-1] <= 1_024 * n_seqs
    n = int(seqs[-1])
    lp = -rng.exponential(size=n).astype(np.float32)
    ref, scores = (lp + rng.normal(0, 0.3, n)).astype(np.float32), rng.normal(size=n_seqs).astype(np.float32)
    for mask in (None, rng.random(n) < 0.8):
        for mean in (False, True):
            _check_preference(T, seqs, lp, ref, mask, scores, groups, 0.01, 0.1, 1.0, mean, f"{count} of {sizes} {mean}")
    inner = groups[1:-1]  # sequences before the first and after the last group
    if len(inner) > 1:
        _check_preference(T, seqs, lp, ref, None, scores, inner, 0.01, 0.0, 1.0, True, "outside")


@pytest.mark.parametrize("value", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("size", [3, 70, 400, 3_000])
def test_centred_advantages_of_special_scores(T, size, value):
    """A NaN or an infinity makes its whole group NaN, centred or standardised, and no other group."""
    scores = np.random.default_rng(size).normal(size=4 * size).astype(np.float32)
    scores[size + size // 2] = value
    groups = np.arange(0, 4 * size + 1, size)
    for flags in (0, T.TREE_ENS_CENTER_ONLY):
        got = T.tree_ens_group_advantage(_dev(scores), _dev(groups), flags=flags).cpu().numpy()
        assert np.isnan(got[size:2 * size]).all() and np.isfinite(np.delete(got, np.s_[size:2 * size])).all()
        want = O.group_advantage(scores, groups, 1e-6, bool(flags))
        assert np.array_equal(np.isnan(got), np.isnan(want))


@pytest.mark.parametrize("count,sizes", [(1_212, [96] * 605 + [2_040]), (1_212, [96] * 605 + [2_500]), (60, [20] * 29 + [700]),
                                         (3_000, [2] * 2_999 + [2_000]), (1, [2_047])])
def test_many_alike_pairs_add_up(T, count, sizes):
    """The best answer of a large group leads all others, which are alike, by the same margin: adding equal terms rounds
    the same way each time. A pair is off by 32 u, and a chain of 128 floats adds 64 u to each at most."""
    groups = np.concatenate([[0], np.cumsum(np.resize(sizes, count))]).astype(np.int64)
    n = int(groups[-1])
    lp, scores = np.zeros(n, np.float32), -np.arange(n, dtype=np.float32)
    for lead in (0.1, 0.3, 0.7, 1.1, 2.3):
        lp[groups[:-1]] = lead
        loss, _, grad = T.tree_ens_preference_loss(_dev(lp), _dev(np.arange(n + 1)), _dev(scores), _dev(groups), beta=1.0)
        for g in range(0, count, max(1, count // 20)) if count > 60 else range(count):
            _alike(loss[g:g + 1], grad[groups[g]:groups[g + 1]], lead, f"group {g}")
        _alike(loss[-1:], grad[groups[-2]:], lead, "last group")


def _alike(loss, grad, lead, what):
    n, d = grad.numel(), float(np.float32(lead))
    pairs = n * (n - 1) / 2
    rank = np.arange(1, n)  # of the others, from the second best on: with r others ahead and n - 1 - r behind
    slope, even = -1 / (1 + np.exp(d)), 0.5
    want = np.concatenate([[(n - 1) * slope], -slope + even * (rank - 1) - even * (n - 1 - rank)]) / pairs
    _close(grad, want, 100 * U * (n - 1) / pairs + 4 * U * np.abs(want), what + " gradient")
    mean = ((n - 1) * np.log1p(np.exp(-d)) + (pairs - (n - 1)) * np.log(2)) / pairs
    _close(loss, np.array([mean]), 100 * U, what + " loss")


@pytest.mark.parametrize("count,sizes", [
    (300, [2] * 99 + [9]), (3_000, [2] * 99 + [9]), (3_000, [1, 2, 3, 20, 30, 2, 3, 1, 2]),  # more candidates than lanes
    (60, [30] * 28 + [513, 1_500]), (700, [10] * 69 + [512]),                                # the windows of a workgroup
])
def test_groups_of_every_size_among_small_ones(T, count, sizes):
    rng = np.random.default_rng([count, len(sizes)])
    groups = np.concatenate([[0], np.cumsum(np.resize(sizes, count))]).astype(np.int64)
    n_seqs = int(groups[-1])
    seqs = np.concatenate([[0], np.cumsum(rng.integers(0, 12, n_seqs))]).astype(np.int64)
    n = int(seqs[-1])
    lp, ref = -rng.exponential(size=n).astype(np.float32), -rng.exponential(size=n).astype(np.float32)
    scores = (np.round(rng.normal(size=n_seqs) * 8) / 8).astype(np.float32)
    for smoothing, mean in ((0.0, False), (0.2, True)):
        _check_preference(T, seqs, lp, ref, rng.random(n) < 0.8, scores, groups, 0.2, smoothing, 1.0, mean, f"{count} of {sizes}")


@pytest.mark.parametrize("count,sizes", [(5_000, [1] * 4_999 + [3_000]), (5_000, [3] * 2_499 + [2_000]), (600, [80] * 99 + [4_000]),
                                         (300, [200] * 99 + [2_049]), (120, [300] * 59 + [9_000])])
def test_advantages_of_a_large_group_among_small_ones(T, count, sizes):
    rng = np.random.default_rng([count, sizes[-1]])
    groups = np.concatenate([[0], np.cumsum(np.resize(sizes, count))]).astype(np.int64)
    scores = (5 + 0.1 * rng.normal(size=int(groups[-1]))).astype(np.float32)
    for flags in (0, T.TREE_ENS_CENTER_ONLY):
        x = _dev(scores)
        got = T.tree_ens_group_advantage(x, _dev(groups), eps=1e-3, flags=flags)
        want = O.group_advantage(scores, groups, float(np.float32(1e-3)), bool(flags))
        _close(got, want, 4 * U * np.abs(want) + 1e-12, f"{count} of {sizes} {flags}")
        T.tree_ens_group_advantage(x, _dev(groups), eps=1e-3, flags=flags, advantages=x)
        assert bool((x == got).all())
