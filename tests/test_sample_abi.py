"""Refusals of sampling, of the gradients' norm and of clipping: every one comes before any HIP call, so they show on a
host without a GPU. Pointers are addresses of host memory that nothing reads as device memory."""
from __future__ import annotations

import ctypes

import numpy as np
import pytest

import paper_1212_2287_amd as T

BUF = np.zeros(4096, np.float64)  # 16-byte aligned stands-in for device memory
P = (BUF.ctypes.data + 15) // 16 * 16


@pytest.fixture(scope="module")
def lib():
    return T.load_library()


def _refused(lib, fn, args, match):
    assert getattr(lib, fn)(*args) == T.TREE_ENS_E_ARG, (fn, args)
    assert match in T.tree_ens_last_error(), T.tree_ens_last_error()


SAMPLE = dict(stream=None, logits=P, dtype=1, n=4, v=8, stride=8, uniform=P, scale=1.0, top_k=0, top_p=1.0, min_p=0.0,
              row_scale=None, row_top_k=None, row_top_p=None, row_min_p=None, tokens=P, logp=P, log_kept=P, work=None,
              work_bytes=0)
NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("change,match", [
    (dict(dtype=3), "dtype"), (dict(dtype=-1), "dtype"), (dict(n=-1), "n_tokens"), (dict(v=0), "n_vocab"),
    (dict(v=2**31), "n_vocab"), (dict(stride=7), "row_stride"), (dict(stride=2**62), "row_stride"),
    (dict(scale=0.0), "scale"), (dict(scale=-1.0), "scale"), (dict(scale=INF), "scale"), (dict(scale=NAN), "scale"),
    (dict(top_k=-1), "top_k"), (dict(top_p=0.0), "top_p"), (dict(top_p=1.5), "top_p"), (dict(top_p=NAN), "top_p"),
    (dict(min_p=-0.1), "min_p"), (dict(min_p=1.1), "min_p"), (dict(min_p=NAN), "min_p"),
    (dict(logits=None), "NULL"), (dict(uniform=None), "NULL"), (dict(tokens=None), "NULL"),
    (dict(logits=P + 1), "misaligned"), (dict(uniform=P + 4), "misaligned"), (dict(tokens=P + 4), "misaligned"),
    (dict(logp=P + 2), "misaligned"), (dict(log_kept=P + 1), "misaligned"), (dict(row_scale=P + 2), "misaligned"),
    (dict(row_top_k=P + 2), "misaligned"), (dict(row_top_p=P + 2), "misaligned"), (dict(row_min_p=P + 2), "misaligned"),
])
def test_sample(lib, change, match):
    _refused(lib, "tree_ens_sample", {**SAMPLE, **change}.values(), match)


def test_sample_workspace(lib):
    need = ctypes.c_int64(-1)
    for n, v in ((0, 1), (1, 1), (8, 100), (1, 200_000), (4_000, 130_000)):
        assert lib.tree_ens_sample_workspace(1, n, v, ctypes.byref(need)) == 0 and need.value >= 0
        if need.value:
            args = {**SAMPLE, "n": n, "v": v, "stride": v}
            _refused(lib, "tree_ens_sample", args.values(), "workspace")
            _refused(lib, "tree_ens_sample", {**args, "work": P, "work_bytes": need.value - 1}.values(), "workspace")
            _refused(lib, "tree_ens_sample", {**args, "work": P + 8, "work_bytes": need.value}.values(), "16-byte")
    _refused(lib, "tree_ens_sample_workspace", (1, 8, 100, None), "NULL")
    _refused(lib, "tree_ens_sample_workspace", (5, 8, 100, ctypes.byref(need)), "dtype")
    _refused(lib, "tree_ens_sample_workspace", (1, -8, 100, ctypes.byref(need)), "n_tokens")
    _refused(lib, "tree_ens_sample_workspace", (1, 8, 0, ctypes.byref(need)), "n_vocab")


def _tensors(*items):
    """(pointers, counts, types) of (address, count, type) items."""
    n = len(items)
    return ((ctypes.c_void_p * n)(*[i[0] for i in items]), (ctypes.c_int64 * n)(*[i[1] for i in items]),
            (ctypes.c_int32 * n)(*[i[2] for i in items]))


def _norm(lib, match, *items, n=None, norm=P, work=P, size=1 << 20):
    p, c, d = _tensors(*items)
    _refused(lib, "tree_ens_grad_norm", (None, len(items) if n is None else n, p, c, d, norm, work, size), match)


def test_grad_norm(lib):
    _norm(lib, "n_tensors", (P, 4, 0), n=-1)
    _norm(lib, "dtypes", (P, 4, 3))
    _norm(lib, "dtypes", (P, 4, 0), (P, 4, -1))
    _norm(lib, "counts", (P, -1, 0))
    _norm(lib, "counts", (P, 2**62, 0))
    _norm(lib, "NULL", (None, 4, 0))
    _norm(lib, "misaligned", (P + 2, 4, 0))
    _norm(lib, "misaligned", (P + 1, 4, 1))
    _norm(lib, "norm", (P, 4, 0), norm=None)
    _norm(lib, "norm", (P, 4, 0), norm=P + 2)
    _norm(lib, "workspace", (P, 4, 0), work=None)
    _norm(lib, "workspace", (P, 4, 0), size=8)
    _norm(lib, "16-byte", (P, 4, 0), work=P + 8)
    _refused(lib, "tree_ens_grad_norm", (None, 1, None, None, None, P, P, 1 << 20), "NULL")
    need = ctypes.c_int64(-1)
    assert lib.tree_ens_grad_norm_workspace(0, ctypes.byref(need)) == 0 and need.value == 0
    assert lib.tree_ens_grad_norm_workspace(700, ctypes.byref(need)) == 0 and need.value > 0
    _refused(lib, "tree_ens_grad_norm_workspace", (-1, ctypes.byref(need)), "n_tensors")
    _refused(lib, "tree_ens_grad_norm_workspace", (1, None), "NULL")


def _clip(lib, match, items, out, norm=P, max_norm=1.0, eps=1e-6):
    p, c, d = _tensors(*items)
    o = (ctypes.c_void_p * len(out))(*out)
    _refused(lib, "tree_ens_grad_clip", (None, len(items), p, c, d, norm, max_norm, eps, o), match)


def test_grad_clip(lib):
    one = [(P, 4, 0)]
    for bad in (dict(max_norm=-1.0), dict(max_norm=NAN), dict(max_norm=INF), dict(eps=-1.0), dict(eps=NAN), dict(eps=INF)):
        _clip(lib, "max_norm", one, [P], **bad)
    _clip(lib, "NULL", one, [P], norm=None)
    _clip(lib, "norm", one, [P], norm=P + 1)
    _clip(lib, "NULL", one, [None])
    _clip(lib, "misaligned", one, [P + 2])
    _clip(lib, "dtypes", [(P, 4, 9)], [P])
    _refused(lib, "tree_ens_grad_clip", (None, 1, *_tensors(*one), P, 1.0, 0.0, None), "NULL")


@pytest.mark.parametrize("items,out", [
    ([(P, 4, 0)], [P + 4]), ([(P, 4, 0)], [P - 4]), ([(P + 64, 4, 1)], [P + 70]),        # over itself, but shifted
    ([(P, 4, 0), (P, 4, 0)], [P, P]),                                                    # the same tensor twice
    ([(P, 4, 0), (P + 64, 4, 0)], [P + 128, P + 140]),                                   # two results
    ([(P, 4, 0), (P + 64, 4, 0)], [P + 64, P + 128]),                                    # onto another's gradient
    ([(P, 4, 0), (P + 64, 4, 0)], [P, P + 12]),
    ([(P, 8, 0), (P + 16, 4, 1)], [P, P + 256]),                                         # gradients that overlap, one in place
])
def test_grad_clip_refuses_overlaps(lib, items, out):
    _clip(lib, "overlaps", items, out)


def test_grad_clip_refuses_the_norm_among_its_results(lib):
    for norm in (P, P + 4, P + 12):
        _clip(lib, "overlaps", [(P, 4, 0)], [P], norm=norm)
        _clip(lib, "overlaps", [(P + 64, 4, 0)], [P], norm=norm)


def test_more_elements_than_numbers_hold(lib):
    many = [(P, 2**47, 0), (P, 2**47, 1), (P, 1, 0)]
    _norm(lib, "counts", *many)
    _clip(lib, "counts", many, [P] * 3)
    _norm(lib, "counts", *[(P, 2**48, 0)] * 9)


def test_nothing_to_do_is_no_error(lib):
    assert lib.tree_ens_sample(*{**SAMPLE, "n": 0, "logits": None, "uniform": None, "tokens": None}.values()) == 0
    assert lib.tree_ens_grad_clip(None, 0, None, None, None, None, 1.0, 1e-6, None) == 0


def test_binding_refuses_host_tensors():
    import torch
    x = torch.zeros(2, 4)
    with pytest.raises(TypeError, match="logits"):
        T.tree_ens_sample(x, torch.zeros(2, dtype=torch.float64))
    with pytest.raises(TypeError, match="CUDA"):
        T.tree_ens_grad_norm([x])
    with pytest.raises(TypeError, match="CUDA"):
        T.tree_ens_grad_clip([x], torch.zeros(()), 1.0)
    for nothing in ([], [None], [x, 3.0]):
        with pytest.raises(TypeError, match="grads"):
            T.tree_ens_grad_norm(nothing)


def test_dense_tensors():
    """Tensors whose elements lie one behind the other in whatever order, and ones with gaps or repeats."""
    import torch

    from paper_1212_2287_amd import _binding as B
    x = torch.zeros(2, 3, 4, 5)
    for t in (x, x.permute(3, 1, 0, 2), x.contiguous(memory_format=torch.channels_last), x[1], x[:, :0], torch.zeros(()),
              torch.zeros(3, 1).expand(3, 1), x[:1], torch.zeros(4, 6).t()):
        assert B._dense(t), t.stride()
    for t in (x[:, 1], x[..., ::2], torch.zeros(1).expand(3), torch.zeros(3, 1).expand(3, 4), x.permute(1, 0, 2, 3)[:2]):
        assert not B._dense(t), t.stride()
