"""The norm of many tensors and their clipping through the C ABI, against the float64 oracle.

Squares are rounded and added in double (2^-53 each time), so the norm is off by its one rounding to float, 2^-24 of it,
and 2^-40 for the sums. A clipped value carries the roundings of norm + eps, the division, the product and to its type."""
from __future__ import annotations

import numpy as np
import pytest

from oracle import sampling as O

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
LEAST = {"f32": 2.0 ** -149, "bf16": 2.0 ** -133, "f16": 2.0 ** -24}  # the smallest value above 0


@pytest.fixture(scope="module")
def T():
    import paper_1212_2287_amd as T
    T.load_library()
    return T


def _torch_dtype(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[name]


def _tensors(sizes, dtypes, seed=0, bucket=None):
    """Device tensors of the sizes, types in turn, on their own or as views into one buffer a type from `bucket` on."""
    import torch
    rng = np.random.default_rng(seed)
    flat = {d: torch.full((sum(sizes) + 16,), 5.0, dtype=_torch_dtype(d), device="cuda") for d in set(dtypes)}
    at = dict.fromkeys(flat, bucket or 0)
    out = []
    for k, n in enumerate(sizes):
        d = dtypes[k % len(dtypes)]
        v = torch.from_numpy(rng.normal(0, rng.choice([1e-3, 0.1, 2.0]), n)).to(_torch_dtype(d))
        if bucket is None:
            out.append(v.cuda())
        else:
            t = flat[d][at[d]:at[d] + n]
            t.copy_(v)
            at[d] += n
            out.append(t)
    return out


def _host(ts):
    return [t.double().cpu().numpy() for t in ts]


def _check_norm(got, want):
    assert abs(got.double().item() - want) <= (U + 2.0 ** -40) * want, (got.item(), want)


def _check_clipped(got, x, norm, limit, eps, dtypes):
    for k, (g, v) in enumerate(zip(got, x)):
        want = O.grad_clip([v], norm, limit, eps)[0]
        d = dtypes[k % len(dtypes)]
        # four roundings in float (the norm's own, norm + eps, the division, the product) and the one to the type
        e = (4.5 * U + HALF_STEP[d]) * np.abs(want) + LEAST[d]
        assert (np.abs(g.double().cpu().numpy() - want) <= e).all(), k


SIZES = [
    [1], [0], [7], [0, 1, 0], [255, 256, 257], [4096], [2047, 2048, 2049, 1], [100_003], [3] * 300, [0] * 130 + [5],
    [1, 1_000_003, 17, 0, 65_536], [64] * 127 + [9], [64] * 128, [64] * 129, [6_000_001, 40],
]


@pytest.mark.parametrize("dtypes", [["f32"], ["bf16"], ["f16"], ["bf16", "f32", "f16"]])
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{max(s)}")
def test_against_the_oracle(T, sizes, dtypes):
    import torch
    print("[grads]", len(sizes), max(sizes), dtypes, flush=True)
    for bucket in (None, 0, 1, 3):
        ts = _tensors(sizes, dtypes, len(sizes), bucket)
        x = _host(ts)
        want = O.grad_norm(x)
        norm = T.tree_ens_grad_norm(ts)
        assert norm.shape == () and norm.dtype == torch.float32
        _check_norm(norm, want)
        assert torch.equal(norm, T.tree_ens_grad_norm(ts))
        got_norm = norm.double().item()
        for limit in (0.37 * want + 1e-3, 3 * want + 1.0):
            limit = float(np.float32(limit))
            out = [torch.full((t.numel() + 5,), -9.0, dtype=t.dtype, device="cuda") for t in ts]
            views = [o[3:3 + t.numel()] for o, t in zip(out, ts)]
            got = T.tree_ens_grad_clip(ts, norm, limit, out=views)
            assert all(g is v for g, v in zip(got, views))
            _check_clipped(got, x, got_norm, limit, float(np.float32(1e-6)), dtypes)
            assert all((o[:3] == -9).all() and (o[3 + t.numel():] == -9).all() for o, t in zip(out, ts))
            assert all(np.array_equal(a, b) for a, b in zip(_host(ts), x))
        for limit in (3 * want + 1.0, 0.5 * want):
            got = T.tree_ens_grad_clip(ts, norm, limit)
            assert all(g is t for g, t in zip(got, ts))
            _check_clipped(ts, x, got_norm, float(np.float32(limit)), float(np.float32(1e-6)), dtypes)
            if limit > want:
                assert all(np.array_equal(a, b) for a, b in zip(_host(ts), x))
        if bucket is not None:  # what lies beside the views
            used = sum(sizes)
            base = ts[0]._base if len(ts) else None
            if base is not None and len(dtypes) == 1:
                assert (base[:bucket] == 5).all() and (base[bucket + used:] == 5).all()


def test_the_largest_and_smallest_values(T):
    import torch
    for v, n in ((3e38, 1), (1e38, 4), (1e-40, 1000), (2e-45, 7), (1e30, 100_000), (1e-30, 100_000)):
        t = torch.full((n,), v, device="cuda")
        want = t[0].double().item() * n ** 0.5
        _check_norm(T.tree_ens_grad_norm([t]), want) if want > 1e-38 else None
        if want <= 1e-38:  # the norm is a subnormal float: half of the smallest
            assert abs(T.tree_ens_grad_norm([t]).double().item() - want) <= 2.0 ** -150 * 1.01
    assert T.tree_ens_grad_norm([torch.full((4,), 3e38, device="cuda")]).item() == np.inf  # 6e38 is no float
    assert T.tree_ens_grad_norm([torch.zeros(9, device="cuda")]).item() == 0.0


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_infinities_and_nan(T, dtype):
    import torch
    base = torch.ones(5000, dtype=_torch_dtype(dtype), device="cuda")
    for at in (0, 1, 2500, 4999):
        for v in (np.inf, -np.inf):
            t = base.clone()
            t[at] = v
            norm = T.tree_ens_grad_norm([base, t])
            assert norm.item() == np.inf
            a, b = T.tree_ens_grad_clip([base.clone(), t], norm, 1.0)
            assert not a.any() and torch.isnan(b[at]) and not b[torch.arange(5000, device="cuda") != at].any()
        t = base.clone()
        t[at] = np.nan
        norm = T.tree_ens_grad_norm([t, base])
        assert torch.isnan(norm)
        assert all(torch.isnan(c).all() for c in T.tree_ens_grad_clip([t, base.clone()], norm, 1.0))


def test_limits_of_clipping(T):
    import torch
    t = torch.tensor([3.0, 4.0], device="cuda")
    norm = T.tree_ens_grad_norm([t])
    assert norm.item() == 5.0
    clip = lambda **kw: T.tree_ens_grad_clip([t], norm, out=[torch.empty_like(t)], **kw)[0].tolist()  # noqa: E731
    assert clip(max_norm=5.0, eps=0.0) == [3.0, 4.0] and clip(max_norm=2.5, eps=0.0) == [1.5, 2.0]
    assert clip(max_norm=0.0) == [0.0, 0.0] and clip(max_norm=10.0, eps=15.0) == [1.5, 2.0]
    zero = torch.zeros(3, device="cuda")
    assert T.tree_ens_grad_clip([zero], T.tree_ens_grad_norm([zero]), 1.0)[0].tolist() == [0.0, 0.0, 0.0]
    nothing = T.tree_ens_grad_norm([torch.empty(0, device="cuda")])
    assert nothing.item() == 0.0


def test_nothing_to_scale_by(T):
    """No norm, no norm allowed and no eps: 0 over 0 leaves the zeros."""
    import torch
    x = [torch.zeros(300, device="cuda"), torch.zeros(7, device="cuda", dtype=torch.bfloat16)]
    out = T.tree_ens_grad_clip(x, T.tree_ens_grad_norm(x), 0.0, eps=0.0, out=[torch.ones_like(t) for t in x])
    assert all(torch.equal(o, t) for o, t in zip(out, x))


def test_many_workgroups_sums(T):
    """More launches' sums than the last kernel has threads times loads."""
    import torch
    x = torch.from_numpy(np.random.default_rng(3).normal(0, 1, (700, 50_000)).astype(np.float32)).cuda()
    _check_norm(T.tree_ens_grad_norm(list(x)), x.double().square().sum().sqrt().item())


def test_the_norm_is_not_clipped(T):
    import torch
    x = torch.ones(100, device="cuda")
    with pytest.raises(T.TreeEnsError, match="overlaps"):
        T.tree_ens_grad_clip([x], x[3:4], 1.0)
    T.tree_ens_grad_clip([x], x[3:4], 1.0, eps=0.0, out=[torch.empty_like(x)])  # read only
    norm = T.tree_ens_grad_norm([x], norm=x[5:6])  # written behind all reads
    assert norm.item() == 10.0 and x[5].item() == 10.0 and x.sum().item() == 109.0


def test_shapes_and_orders_of_dimensions(T):
    import torch
    g = torch.Generator(device="cuda").manual_seed(0)
    x = torch.randn(6, 5, 4, 3, generator=g, device="cuda")
    ts = [x, x.permute(3, 0, 2, 1), x.contiguous(memory_format=torch.channels_last), torch.tensor(2.0, device="cuda"), x[2].t() if x[2].dim() == 2 else x[2, 0].t()]
    want = O.grad_norm(_host(ts))
    _check_norm(T.tree_ens_grad_norm(ts), want)
    norm = T.tree_ens_grad_norm(ts)
    out = T.tree_ens_grad_clip(ts, norm, 1.0, out=[torch.empty_like(t) for t in ts])
    for o, t in zip(out, ts):
        assert torch.allclose(o, t * (1.0 / (norm + 1e-6)), rtol=4 * U, atol=0)
    assert T.tree_ens_grad_norm(t for t in ts).item() == norm.item()  # any sequence
    twice = T.tree_ens_grad_norm([x, x])
    _check_norm(twice, 2 ** 0.5 * O.grad_norm(_host([x])))
    for bad in (x[:, 1], x[..., ::2], x[:1].expand(2, 5, 4, 3)):
        with pytest.raises(TypeError, match="gaps"):
            T.tree_ens_grad_norm([x, bad])
    for bad in ([x.double()], [x.long()]):
        with pytest.raises(TypeError, match="float32"):
            T.tree_ens_grad_norm(bad)
    with pytest.raises(TypeError, match="one device"):
        T.tree_ens_grad_norm([x, x.cpu()])
    with pytest.raises(TypeError, match="norm"):
        T.tree_ens_grad_norm([x], norm=torch.empty(2, device="cuda"))
    with pytest.raises(TypeError, match="norm"):
        T.tree_ens_grad_clip([x], 3.0, 1.0)
    with pytest.raises(TypeError, match="out"):
        T.tree_ens_grad_clip([x], norm, 1.0, out=[])
    for bad in (x[0], x.bfloat16(), torch.empty(3, 4, 5, 6, device="cuda").permute(3, 2, 1, 0)):
        with pytest.raises(TypeError, match="out"):
            T.tree_ens_grad_clip([x], norm, 1.0, out=[bad])
    with pytest.raises(T.TreeEnsError, match="overlaps"):
        T.tree_ens_grad_clip([x, x], norm, 1.0)
    with pytest.raises(T.TreeEnsError, match="max_norm"):
        T.tree_ens_grad_clip([x], norm, -1.0)


def test_more_than_2_31_elements(T):
    import torch
    n = 2 ** 31 + 4097
    t = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    for at, v in ((0, 3.0), (2 ** 31 - 1, 4.0), (2 ** 31 + 4096, 12.0)):
        t[at] = v
    norm = T.tree_ens_grad_norm([t, torch.full((3,), 0.0, device="cuda")])
    assert norm.item() == 13.0
    T.tree_ens_grad_clip([t], norm, 6.5, eps=0.0)
    assert [t[at].item() for at in (0, 2 ** 31 - 1, 2 ** 31 + 4096)] == [1.5, 2.0, 6.0] and t.count_nonzero().item() == 3


def test_another_stream_and_equal_bits(T):
    import torch
    ts = _tensors([100_001, 7, 3_000_000], ["bf16", "f32"])
    side = torch.cuda.Stream()
    first = T.tree_ens_grad_norm(ts)
    want = T.tree_ens_grad_clip(ts, first, 1.0, out=[torch.empty_like(t) for t in ts])
    side.wait_stream(torch.cuda.current_stream())
    for stream in (side, side.cuda_stream):
        norm = T.tree_ens_grad_norm(ts, stream=stream)
        got = T.tree_ens_grad_clip(ts, norm, 1.0, out=[torch.empty_like(t) for t in ts], stream=stream)
        side.synchronize()
        assert torch.equal(norm, first) and all(torch.equal(a, b) for a, b in zip(got, want))


def test_captured_into_a_graph(T):
    """More tensors than one launch takes; replays go by the tensors' present values and find the same places."""
    import torch
    ts = _tensors([500] * 200 + [70_001], ["f32", "bf16"])
    out = [torch.empty_like(t) for t in ts]
    norm = torch.empty((), device="cuda")

    def step():
        T.tree_ens_grad_norm(ts, norm=norm)
        T.tree_ens_grad_clip(ts, norm, 1.0, out=out)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for _ in range(2):  # two graphs, each with a workspace of its own
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            step()
    for k in range(3):
        for t in ts:
            t.normal_(0, 0.1 + k)
        step()
        want = [norm.clone()] + [o.clone() for o in out]
        for graph in graphs:
            for o in [norm, *out]:
                o.fill_(-7.0)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip([norm, *out], want)), k


def test_gradients_of_a_model(T):
    """[p.grad for p in parameters] against torch's own clipping, in float64."""
    import torch
    torch.manual_seed(0)
    model = torch.nn.Sequential(torch.nn.Linear(50, 64), torch.nn.Tanh(), torch.nn.Linear(64, 8)).cuda()
    model(torch.randn(20, 50, device="cuda")).square().sum().backward()
    grads = [p.grad for p in model.parameters()]
    ref = [torch.nn.Parameter(g.double()) for g in grads]
    for r, g in zip(ref, grads):
        r.grad = g.double()
    want = torch.nn.utils.clip_grad_norm_(ref, 0.5)
    norm = T.tree_ens_grad_norm(grads)
    _check_norm(norm, want.item())
    T.tree_ens_grad_clip(grads, norm, 0.5)
    for p, r in zip(model.parameters(), ref):
        assert torch.allclose(p.grad.double(), r.grad, rtol=6 * U, atol=0)
