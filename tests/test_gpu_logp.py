"""GPU token log-probabilities and their gradient through the C ABI, against the float64 oracle on the same
(already rounded) logits.

Tolerances, with u = 2^-24 and K = V / 256 + 64 additions on a value's way into a sum (each rounds the sum by at
most u): z = scale * (x - max) is rounded twice, exp2 of it is off by 4u (1 + |z|), the sum S by (K + 4) u
relative, so log S absolutely; the entropy adds W / S <= log S + entropy with the same relative error."""
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


def _torch_dtype(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[name]


def _logits(dtype, n, V, pad=0, first=0, seed=0, banned=0.0):
    """Device logits [n, V] with rows V + pad apart, the first one `first` elements into its allocation, and
    the values they stand for."""
    import torch
    rng = np.random.default_rng([seed, n, V])
    x = rng.normal(0, 3, (n, V))
    x[np.arange(n), rng.integers(0, V, n)] += 8
    if banned:
        x[:, rng.random(V) < banned] = -np.inf
    flat = torch.zeros(first + n * (V + pad), dtype=_torch_dtype(dtype), device="cuda")
    d = flat[first:].view(n, V + pad)[:, :V]
    d.copy_(torch.from_numpy(x))
    t = rng.integers(0, V, n)
    t[rng.random(n) < 0.2] = -100
    return d, torch.from_numpy(t).cuda(), d.double().cpu().numpy(), t


def _forward_tolerance(V, logp, entropy, stats):
    K = V / 256 + 64
    L, z = np.abs(stats[:, 1]), np.abs(np.nan_to_num(logp, neginf=0.0))
    return U * (4 * (1 + z + L) + K + 8), U * (K + 16) * (1 + 2 * L + entropy), U * (4 * (1 + L) + K + 8)


def _check_forward(got, want, V, what):
    logp, entropy, stats = (g.double().cpu().numpy() for g in got)
    tol = _forward_tolerance(V, *want)
    assert np.array_equal(stats[:, 0], want[2][:, 0]), what
    for name, a, b, e in (("logp", logp, want[0], tol[0]), ("entropy", entropy, want[1], tol[1]),
                          ("log sum", stats[:, 1], want[2][:, 1], tol[2])):
        fine = np.isfinite(b)
        assert np.array_equal(a[~fine], b[~fine]), (what, name)
        err = np.abs(a[fine] - b[fine]) / e[fine]
        assert (err <= 1).all(), (what, name, float(err.max()))


def _grad_tolerance(want, x, t, g, h, scale, dtype, stats, entropy):
    z = scale * (x - x.max(1, keepdims=True))
    l = z - stats[:, 1:]
    p = np.exp(l)
    l = np.where(p > 0, l, 0.0)
    z = np.where(p > 0, z, 0.0)
    g, h, H = np.abs(g)[:, None], np.abs(h)[:, None], np.abs(entropy)[:, None]
    rel = U * (8 + 6 * np.abs(z) + 4 * np.abs(stats[:, 1:]))  # of p
    e = scale * (rel * p * (g + h * (np.abs(l) + H)) + p * U * 8 * (g + h * (np.abs(l) + H)) + 2 * U * g * (np.arange(x.shape[1]) == t[:, None]))
    step, least = {"f32": (U, 2.0 ** -126), "bf16": (2.0 ** -9, 2.0 ** -126), "f16": (2.0 ** -12, 2.0 ** -25)}[dtype]
    return e + 2 * step * np.abs(want) + least


def _check_backward(T, dtype, d, td, x, t, scale, seed, what, entropies=True, **kw):
    import torch
    rng = np.random.default_rng(seed)
    n = len(t)
    g, h = rng.normal(size=n).astype(np.float32), rng.normal(size=n).astype(np.float32)
    g[rng.random(n) < 0.2] = 0.0
    if not entropies:
        h[:] = 0.0
    logp, entropy, stats = O.token_logp(x, t, scale)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.float32)).cuda()  # noqa: E731
    more = dict(entropy=dev(entropy), grad_entropy=dev(h)) if entropies else {}
    out = T.tree_ens_token_logp_backward(d, td, dev(stats), dev(g), scale=scale, **more, **kw)
    assert out.dtype == d.dtype
    got = out.double().cpu().numpy()
    want = O.token_logp_grad(x, t, g, h, scale)
    tol = _grad_tolerance(want, x, t, g, h, scale, dtype, stats, entropy)
    err = np.abs(got - want) / tol
    assert (err <= 1).all(), (what, float(err.max()), np.argwhere(err > 1)[:3].tolist())
    return out


SHAPES = [
    # tokens, vocabulary, padding of a row, elements before the first row
    (1, 1, 0, 0), (3, 2, 0, 0), (5, 7, 1, 1), (9, 63, 0, 0), (4, 64, 0, 0), (300, 65, 0, 3), (17, 255, 2, 0), (8, 257, 0, 1),
    (70, 1000, 0, 0), (33, 1023, 0, 0), (6, 2047, 2, 5), (5, 2048, 0, 0), (3, 2049, 7, 0), (2, 4097, 0, 0), (4, 8192, 8, 0),
    (1, 20_001, 0, 0), (3, 32_000, 0, 0), (2, 65_537, 0, 1), (1, 131_072, 0, 0), (40, 50_001, 0, 0),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,V,pad,first", SHAPES)
def test_against_the_oracle(T, dtype, n, V, pad, first):
    what = f"{dtype} {n} x {V} + {pad} from {first}"
    print("[logp]", what, flush=True)
    for scale, banned in ((1.0, 0.0), (0.6, 0.4)):
        d, td, x, t = _logits(dtype, n, V, pad, first, seed=1, banned=banned)
        live = np.where((t >= 0) & (t < V), t, 0)
        if V > 1:  # the target may be banned; the row keeps something
            d[:, 0] = 1.0
            x[:, 0] = 1.0
        got = T.tree_ens_token_logp(d, td, scale=scale, want_entropy=True)
        _check_forward(got, O.token_logp(x, t, scale), V, what)
        plain = T.tree_ens_token_logp(d, td, scale=scale)
        assert plain[1] is None
        _check_forward((plain[0], got[1], plain[2]), O.token_logp(x, t, scale), V, what + " without entropy")
        if np.isfinite(x).any(1).all():
            _check_backward(T, dtype, d, td, x, t, scale, 2, what)
            _check_backward(T, dtype, d, td, x, t, scale, 3, what + " without entropy", entropies=False)
        assert (live < V).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V", [5, 300, 3000, 40_000])
def test_rows_of_special_values(T, dtype, V):
    import torch
    lowest = torch.finfo(_torch_dtype(dtype)).min
    n = 10
    x = np.random.default_rng(V).normal(0, 2, (n, V))
    x[0] = -np.inf                     # nothing can be sampled
    x[1] = -np.inf
    x[1, V - 1] = 2.0                  # one token, the target
    x[2] = -np.inf
    x[2, 1] = -3.0                     # one token, not the target
    x[3] = lowest                      # masked by the lowest value, all alike
    x[4] = lowest
    x[4, V - 1] = 0.5
    x[5, 2] = np.nan
    x[6, V // 2] = np.inf
    x[7] = 0.0
    t = np.array([V - 1] * 8 + [V, -1])
    d = torch.from_numpy(x).to(_torch_dtype(dtype)).cuda()
    td = torch.from_numpy(t).cuda()
    x = d.double().cpu().numpy()
    logp, entropy, stats = (a.double().cpu().numpy() for a in T.tree_ens_token_logp(d, td, want_entropy=True))
    fine = [0, 1, 2, 3, 4, 7, 8, 9]
    want = O.token_logp(x, t)
    _check_forward([torch.from_numpy(a[fine]) for a in (logp, entropy, stats)], [w[fine] for w in want], V, "special rows")
    assert logp[0] == -np.inf and entropy[0] == 0 and logp[2] == -np.inf and logp[1] == 0 and entropy[1] == 0
    assert np.isnan(logp[[5, 6]]).all() and np.isnan(entropy[[5, 6]]).all()
    assert not logp[8:].any() and not stats[8:].any()
    g = torch.ones(n, device="cuda")
    f32 = lambda a: torch.from_numpy(a).float().cuda()  # noqa: E731
    for h in (None, torch.ones(n, device="cuda")):
        got = T.tree_ens_token_logp_backward(d, td, f32(stats), g, entropy=f32(entropy) if h is not None else None,
                                             grad_entropy=h).double().cpu().numpy()
        ones = np.ones(n)
        ref = np.zeros((n, V))
        ref[fine] = O.token_logp_grad(x[fine], t[fine], ones[fine], None if h is None else ones[fine])
        tol = _grad_tolerance(ref[1:5], x[1:5], t[1:5], ones[1:5], ones[1:5], 1.0, dtype, want[2][1:5], want[1][1:5])
        assert (np.abs(got[1:5] - ref[1:5]) <= tol).all()
        assert not got[0].any() and not got[8:].any()
        assert np.isnan(got[[5, 6]]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,V,pad", [(7, 1001, 3), (3, 20_001, 0)])
def test_gradient_in_place_of_the_logits_and_into_padded_rows(T, dtype, n, V, pad):
    import torch
    d, td, x, t = _logits(dtype, n, V, pad, 1)
    wide = torch.full((n, V + 5), 7.0, dtype=d.dtype, device="cuda")
    _check_backward(T, dtype, d, td, x, t, 1.0, 4, "padded", grad_logits=wide[:, 2:V + 2])
    assert (wide[:, :2] == 7).all() and (wide[:, V + 2:] == 7).all()
    around = d.as_strided((n - 1, pad), (V + pad, 1), d.storage_offset() + V).clone()
    out = _check_backward(T, dtype, d, td, x, t, 1.0, 4, "in place", grad_logits=d)
    assert out.data_ptr() == d.data_ptr()
    assert torch.equal(around, d.as_strided((n - 1, pad), (V + pad, 1), d.storage_offset() + V))


def test_gradient_by_differences(T):
    """grad_logits against differences of the float64 oracle's forward along random directions: the gradient is of
    float32 accuracy, the difference of a step of 1e-4 has an error of about 1e-8."""
    import torch
    rng = np.random.default_rng(8)
    n, V = 6, 501
    d, td, x, t = _logits("f32", n, V)
    g, h = rng.normal(size=n).astype(np.float32), rng.normal(size=n).astype(np.float32)
    _, entropy, stats = T.tree_ens_token_logp(d, td, scale=1.3, want_entropy=True)
    grad = T.tree_ens_token_logp_backward(d, td, stats, torch.from_numpy(g).cuda(), scale=1.3, entropy=entropy,
                                          grad_entropy=torch.from_numpy(h).cuda()).double().cpu().numpy()
    for _ in range(4):
        u = rng.normal(size=(n, V))

        def f(e):
            a, b, _ = O.token_logp(x + e * u, t, 1.3)
            return (g * a + h * b * ((t >= 0) & (t < V))).sum()
        assert abs((f(1e-4) - f(-1e-4)) / 2e-4 - (grad * u).sum()) < 2e-4


def test_another_stream_and_equal_bits(T):
    import torch
    d, td, x, t = _logits("bf16", 37, 30_011)
    side = torch.cuda.Stream()
    first = T.tree_ens_token_logp(d, td, want_entropy=True)
    side.wait_stream(torch.cuda.current_stream())
    again = T.tree_ens_token_logp(d, td, want_entropy=True, stream=side)
    raw = T.tree_ens_token_logp(d, td, want_entropy=True, stream=side.cuda_stream)
    side.synchronize()
    for a, b, c in zip(first, again, raw):
        assert torch.equal(a, b) and torch.equal(a, c)


def test_offsets_past_32_bits(T):
    """Rows whose logits lie beyond 2^31 elements (and 2^32 bytes) of the first."""
    import torch
    n, V, stride = 5, 1000, 600_000_000
    flat = torch.empty((n - 1) * stride + V, dtype=torch.bfloat16, device="cuda")
    d = flat.as_strided((n, V), (stride, 1))
    x = torch.from_numpy(np.random.default_rng(0).normal(0, 2, (n, V))).to(torch.bfloat16)
    d.copy_(x)
    t = np.arange(n)
    _check_forward(T.tree_ens_token_logp(d, torch.from_numpy(t).cuda(), want_entropy=True), O.token_logp(x.double().numpy(), t), V, "far rows")
    _check_backward(T, "bf16", d, torch.from_numpy(t).cuda(), x.double().numpy(), t, 1.0, 1, "far rows", grad_logits=d)


def test_captured_into_a_graph(T):
    import torch
    d, td, _, _ = _logits("f32", 3, 60_001)
    g = torch.randn(3, device="cuda")
    out = [torch.empty(3, device="cuda"), torch.empty(3, device="cuda"), torch.empty(3, 2, device="cuda"), torch.empty_like(d)]

    def step():
        T.tree_ens_token_logp(d, td, logp=out[0], entropy=out[1], stats=out[2])
        T.tree_ens_token_logp_backward(d, td, out[2], g, grad_logits=out[3])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(3):
        d.copy_(torch.randn(d.shape, generator=torch.Generator().manual_seed(k)))
        step()
        want = [o.clone() for o in out]
        for o in out:
            o.fill_(-7.0)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b), k


def test_argument_errors(T):
    import torch
    d, td, _, _ = _logits("f32", 3, 8)
    with pytest.raises(TypeError, match="targets"):
        T.tree_ens_token_logp(d, td.int())
    with pytest.raises(TypeError, match="targets"):
        T.tree_ens_token_logp(d, td[:2])
    with pytest.raises(TypeError, match="contiguous rows"):
        T.tree_ens_token_logp(d.t(), td)
    with pytest.raises(TypeError, match="logits"):
        T.tree_ens_token_logp(d.double(), td)
    with pytest.raises(T.TreeEnsError) as ei:
        T.tree_ens_token_logp(d, td, scale=0.0)
    assert ei.value.code == T.TREE_ENS_E_ARG
    with pytest.raises(T.TreeEnsError):
        T.tree_ens_token_logp(d[:1].expand(3, 8), td)  # rows that share their logits
    _, _, stats = T.tree_ens_token_logp(d, td)
    g = torch.ones(3, device="cuda")
    with pytest.raises(TypeError, match="grad_logp"):
        T.tree_ens_token_logp_backward(d, td, stats, torch.ones(1, device="cuda").expand(3))
    with pytest.raises(TypeError, match="together"):
        T.tree_ens_token_logp_backward(d, td, stats, g, entropy=g)
    with pytest.raises(TypeError, match="grad_logits"):
        T.tree_ens_token_logp_backward(d, td, stats, g, grad_logits=torch.empty(3, 8, device="cuda", dtype=torch.bfloat16))
    empty = torch.empty(0, 8, device="cuda")
    logp, _, _ = T.tree_ens_token_logp(empty, td[:0])
    assert logp.shape == (0,)
    assert T.tree_ens_token_logp_backward(empty, td[:0], torch.empty(0, 2, device="cuda"), g[:0]).shape == (0, 8)


@pytest.mark.parametrize("dtype,n,V,pad", [
    ("bf16", 9_000, 203, 0), ("bf16", 8_200, 2_000, 0), ("f32", 8_001, 1_000, 3),   # 16 threads a row
    ("f16", 2_500, 3_001, 0), ("f32", 20_000, 1_100, 0), ("bf16", 50, 400, 0),      # a wave
    ("bf16", 700, 40_003, 0), ("f32", 20, 1_500, 0), ("f32", 4_100, 17_001, 1),     # 256 threads
    ("bf16", 300, 8_001, 0), ("f16", 130, 60_000, 0),                               # 1,024 threads
    ("bf16", 128, 33_000, 0), ("f32", 2, 200_001, 0), ("f16", 64, 100_001, 7),      # shares of a row
])
def test_every_way_to_split_the_rows(T, dtype, n, V, pad):
    """Rows enough (or few enough) for each way the passes are split, 40 of them against the oracle."""
    print("[logp]", dtype, n, V, pad, flush=True)
    import torch
    d, td, _, t = _logits(dtype, n, V, pad, seed=5)
    pick = np.unique(np.concatenate([[0, n - 1], np.random.default_rng(n).integers(0, n, 38)]))
    x = d[torch.from_numpy(pick).cuda()].double().cpu().numpy()
    want = O.token_logp(x, t[pick], 0.8)
    for entropy in (True, False):
        got = T.tree_ens_token_logp(d, td, scale=0.8, want_entropy=entropy)
        at = [a.cpu()[pick] for a in (got[0], got[1] if entropy else torch.from_numpy(_full(want[1], pick, n)), got[2])]
        _check_forward(at, want, V, f"{dtype} {n} x {V}")
        again = T.tree_ens_token_logp(d, td, scale=0.8, want_entropy=entropy)
        assert torch.equal(got[0], again[0]) and torch.equal(got[2], again[2])
    rng = np.random.default_rng(1)
    g, h = rng.normal(size=n).astype(np.float32), rng.normal(size=n).astype(np.float32)
    _, entropy, stats = T.tree_ens_token_logp(d, td, scale=0.8, want_entropy=True)
    dev = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    for k, more in enumerate(({}, dict(entropy=entropy, grad_entropy=dev(h)))):
        out = T.tree_ens_token_logp_backward(d, td, stats, dev(g), scale=0.8, **more)
        ref = O.token_logp_grad(x, t[pick], g[pick], h[pick] if k else None, 0.8)
        # the statistics are the kernel's: they carry its own rounding
        slack = _forward_tolerance(V, *want)
        tol = _grad_tolerance(ref, x, t[pick], g[pick], h[pick] * k, 0.8, dtype, want[2], want[1])
        p = np.exp(0.8 * (x - x.max(1, keepdims=True)) - want[2][:, 1:])
        tol = tol + 0.8 * p * (np.abs(g[pick]) * slack[2] + k * np.abs(h[pick]) * (slack[1] + slack[2] * (2 + want[1] + np.abs(want[2][:, 1]))))[:, None] * 2
        err = np.abs(out[torch.from_numpy(pick).cuda()].double().cpu().numpy() - ref) / tol
        assert (err <= 1).all(), float(err.max())
        dead = torch.from_numpy((t < 0)).cuda()
        assert not bool(out[dead].any())


def _full(values, pick, n):
    out = np.zeros(n)
    out[pick] = values
    return out


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [60, 900, 5_000])
def test_gradients_of_any_size_leave_excluded_tokens_at_zero(T, dtype, V):
    """Gradients of the entropy (and of the log-probability) up to 1e35: logits of -inf have gradient 0 all the same, the
    others are as large as they are."""
    import torch
    d, td, x, t = _logits(dtype, 6, V, seed=3, banned=0.4)
    d[:, 0] = x[:, 0] = 1.0
    h = np.array([5e8, -1e12, 1e35, 0.0, 1.0, -1e35], np.float32)
    g = np.array([1.0, 1.0, 1.0, 1e30, -1e30, 0.0], np.float32)
    for scale in (1.0, 1.7):
        _, entropy, stats = O.token_logp(x, t, scale)
        dev = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.float32)).cuda()  # noqa: E731
        for k, more in enumerate(({}, dict(entropy=dev(entropy), grad_entropy=dev(h)))):
            out = T.tree_ens_token_logp_backward(d, td, dev(stats), dev(g), scale=scale, **more).double().cpu().numpy()
            want = O.token_logp_grad(x, t, g, h * k, scale)
            tol = _grad_tolerance(want, x, t, g.astype(np.float64), k * h.astype(np.float64), scale, dtype, stats, entropy)
            assert not out[np.isneginf(x) & (np.arange(V) != t[:, None])].any()
            assert (np.abs(out - want) <= tol).all()


def test_entropy_of_a_vocabulary_masked_by_the_lowest_value(T):
    """800 million logits of bfloat16's lowest value and one of 0: its token is certain."""
    import torch
    V = 800_000_000
    d = torch.full((1, V), torch.finfo(torch.bfloat16).min, dtype=torch.bfloat16, device="cuda")
    d[0, V - 5] = 0.0
    logp, entropy, stats = T.tree_ens_token_logp(d, torch.tensor([V - 5], device="cuda"), want_entropy=True)
    assert (logp.item(), entropy.item(), stats.tolist()) == (0.0, 0.0, [[0.0, 0.0]])


def test_scales_up_to_the_largest_float(T):
    """Any finite scale > 0: at 3e38 the largest logit takes everything, and log2(e) times the scale is no float."""
    import torch
    x = np.array([[3.0, 2.5, 2.5, 2.25], [2.5, 3.0, 3.0, 2.5], [2.5, 2.25, 3.0, -np.inf]])
    t = np.array([0, 2, 1])
    d, td, scale = torch.from_numpy(x).float().cuda(), torch.from_numpy(t).cuda(), float(np.float32(3e38))
    want = O.token_logp(x, t, scale)
    got = T.tree_ens_token_logp(d, td, scale=scale, want_entropy=True)
    _check_forward(got, want, 4, "scale 3e38")
    g, h = torch.full((3,), 0.25, device="cuda"), torch.full((3,), 0.125, device="cuda")
    out = T.tree_ens_token_logp_backward(d, td, got[2], g, scale=scale, entropy=got[1], grad_entropy=h).double().cpu().numpy()
    ref = O.token_logp_grad(x, t, np.full(3, 0.25), np.full(3, 0.125), scale)
    assert (np.abs(out - ref) <= 32 * U * scale).all()


def test_gradient_handed_on_to_autograd(T):
    """Outputs carry no graph, and logits.backward(grad_logits) reaches the weights behind the logits as autograd's own
    log_softmax does."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(0)
    hidden = torch.randn(40, 16, generator=g, device="cuda")
    weight = torch.randn(16, 300, generator=g, device="cuda", requires_grad=True)
    t = torch.randint(0, 300, (40,), generator=g, device="cuda")
    grad_logp = torch.randn(40, generator=g, device="cuda")
    logits = hidden @ weight
    logp, _, stats = T.tree_ens_token_logp(logits, t)
    assert not logp.requires_grad and not stats.requires_grad
    logits.backward(T.tree_ens_token_logp_backward(logits, t, stats, grad_logp))
    got, weight.grad = weight.grad, None
    wide = (hidden.double() @ weight.detach().double()).requires_grad_()
    (torch.log_softmax(wide, 1).gather(1, t[:, None])[:, 0] * grad_logp).sum().backward()
    # logits of 16 products are off by 16 u of about 30, and the gradient as much; 40 of them are added
    assert torch.allclose(got.double(), hidden.double().t() @ wide.grad, rtol=0, atol=1e-3)
