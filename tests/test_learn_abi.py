"""Refusals of the operators that learn from scores: every one comes before any HIP call, so they show
on a host without a GPU. Pointers are addresses of host memory that nothing reads."""
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


LOGP = dict(stream=None, logits=P, dtype=1, n=4, v=8, stride=8, targets=P, scale=1.0, logp=P, entropy=None, stats=None,
            work=None, work_bytes=0)


@pytest.mark.parametrize("change,match", [
    (dict(dtype=3), "dtype"), (dict(dtype=-1), "dtype"), (dict(n=-1), "n_tokens"), (dict(v=0), "n_vocab"),
    (dict(v=2**31), "n_vocab"), (dict(stride=7), "row_stride"), (dict(stride=2**62), "row_stride"),
    (dict(scale=0.0), "scale"), (dict(scale=-1.0), "scale"), (dict(scale=float("inf")), "scale"),
    (dict(scale=float("nan")), "scale"), (dict(logits=None), "NULL"), (dict(targets=None), "NULL"), (dict(logp=None), "NULL"),
    (dict(logits=P + 1), "misaligned"), (dict(targets=P + 4), "misaligned"), (dict(logp=P + 2), "misaligned"),
    (dict(entropy=P + 2), "misaligned"), (dict(stats=P + 4), "misaligned"),
])
def test_token_logp(lib, change, match):
    _refused(lib, "tree_ens_token_logp", {**LOGP, **change}.values(), match)


BACK = dict(stream=None, logits=P, dtype=2, n=4, v=8, stride=8, targets=P, scale=1.0, stats=P, grad_logp=P, entropy=None,
            grad_entropy=None, grad=P + 256, grad_stride=8)


@pytest.mark.parametrize("change,match", [
    (dict(dtype=7), "dtype"), (dict(stats=None), "NULL"), (dict(grad_logp=None), "NULL"), (dict(grad=None), "NULL"),
    (dict(grad_stride=7), "grad_stride"), (dict(entropy=P), "both"), (dict(grad_entropy=P), "both"),
    (dict(stats=P + 4), "misaligned"), (dict(grad=P + 257), "misaligned"), (dict(grad=P + 2), "overlaps"),
    (dict(grad=P, grad_stride=9), "overlaps"), (dict(grad=P + 62), "overlaps"),
])
def test_token_logp_backward(lib, change, match):
    _refused(lib, "tree_ens_token_logp_backward", {**BACK, **change}.values(), match)


PREF = dict(stream=None, logp=P, ref=P, mask=P, n=8, seqs=P, n_seqs=4, scores=P, groups=P, n_groups=2, beta=0.1,
            smoothing=0.0, grad_scale=1.0, flags=0, loss=P, margins=P, grad=P, work=P, work_bytes=4096)


@pytest.mark.parametrize("change,match", [
    (dict(n=-1), "n_tokens"), (dict(n_seqs=-1), "counts"), (dict(n_groups=2**31), "counts"),
    (dict(beta=float("nan")), "beta"), (dict(grad_scale=float("inf")), "grad_scale"), (dict(smoothing=1.0), "smoothing"),
    (dict(smoothing=-0.1), "smoothing"), (dict(smoothing=float("nan")), "smoothing"), (dict(flags=2), "flag"),
    (dict(logp=None), "NULL"), (dict(seqs=None), "NULL"), (dict(scores=None), "NULL"), (dict(margins=None), "NULL"),
    (dict(groups=None), "NULL"), (dict(loss=None), "NULL"), (dict(seqs=P + 4), "misaligned"), (dict(ref=P + 1), "misaligned"),
    (dict(work=None), "workspace"), (dict(work_bytes=8), "workspace"), (dict(work=P + 8), "16-byte"),
])
def test_preference_loss(lib, change, match):
    _refused(lib, "tree_ens_preference_loss", {**PREF, **change}.values(), match)


ADV = dict(stream=None, scores=P, n=8, groups=P, n_groups=2, eps=1e-6, flags=0, out=P)


@pytest.mark.parametrize("change,match", [
    (dict(n=-1), "counts"), (dict(n_groups=-1), "counts"), (dict(eps=0.0), "eps"), (dict(eps=float("nan")), "eps"),
    (dict(flags=1), "flag"), (dict(scores=None), "NULL"), (dict(out=None), "NULL"), (dict(groups=None), "NULL"),
    (dict(out=P + 2), "misaligned"),
])
def test_group_advantage(lib, change, match):
    _refused(lib, "tree_ens_group_advantage", {**ADV, **change}.values(), match)


POL = dict(stream=None, logp=P, old=P, ref=P, mask=None, n=8, seqs=P, n_seqs=4, adv=P, low=0.2, high=0.2, kl_coef=0.1,
           grad_scale=1.0, flags=1, loss=P, kl=P, grad=P, work=P, work_bytes=4096)


@pytest.mark.parametrize("change,match", [
    (dict(n=-1), "n_tokens"), (dict(n_seqs=2**31), "counts"), (dict(low=-0.1), "clip_low"), (dict(low=1.1), "clip_low"),
    (dict(high=-0.1), "clip_high"), (dict(high=float("inf")), "clip_high"), (dict(kl_coef=float("nan")), "kl_coef"),
    (dict(ref=None), "ref_logp"), (dict(flags=2), "flag"), (dict(adv=None), "NULL"), (dict(loss=None), "NULL"),
    (dict(logp=None), "NULL"), (dict(old=P + 2), "misaligned"), (dict(kl=P + 1), "misaligned"),
])
def test_policy_loss(lib, change, match):
    _refused(lib, "tree_ens_policy_loss", {**POL, **change}.values(), match)


def test_workspace_sizes(lib):
    need = ctypes.c_int64(-1)
    assert lib.tree_ens_token_logp_workspace(1, 8, 100, ctypes.byref(need)) == 0 and need.value >= 0
    assert lib.tree_ens_preference_workspace(100, 8, 2, ctypes.byref(need)) == 0 and need.value >= 0
    assert lib.tree_ens_policy_workspace(100, 8, ctypes.byref(need)) == 0 and need.value >= 0
    _refused(lib, "tree_ens_token_logp_workspace", (1, 8, 100, None), "NULL")
    _refused(lib, "tree_ens_token_logp_workspace", (5, 8, 100, ctypes.byref(need)), "dtype")
    _refused(lib, "tree_ens_token_logp_workspace", (1, -8, 100, ctypes.byref(need)), "n_tokens")
    _refused(lib, "tree_ens_preference_workspace", (-1, 8, 2, ctypes.byref(need)), "n_tokens")
    _refused(lib, "tree_ens_preference_workspace", (1, 8, 2, None), "NULL")
    _refused(lib, "tree_ens_policy_workspace", (1, -8, ctypes.byref(need)), "counts")
    _refused(lib, "tree_ens_policy_workspace", (1, 8, None), "NULL")


def test_nothing_to_do_is_no_error(lib):
    assert lib.tree_ens_token_logp(*{**LOGP, "n": 0, "logits": None, "targets": None, "logp": None}.values()) == 0
    assert lib.tree_ens_token_logp_backward(*{**BACK, "n": 0, "logits": None}.values()) == 0
    assert lib.tree_ens_group_advantage(*{**ADV, "n": 0, "scores": None, "out": None}.values()) == 0


def test_binding_refuses_host_tensors():
    import torch
    x, t = torch.zeros(2, 4), torch.zeros(2, dtype=torch.int64)
    with pytest.raises(TypeError, match="logits"):
        T.tree_ens_token_logp(x, t)
    with pytest.raises(TypeError, match="logits"):
        T.tree_ens_token_logp_backward(x, t, torch.zeros(2, 2), torch.zeros(2))
    off = torch.tensor([0, 2])
    with pytest.raises(TypeError, match="logp"):
        T.tree_ens_preference_loss(torch.zeros(2), off, torch.zeros(1), off)
    with pytest.raises(TypeError, match="scores"):
        T.tree_ens_group_advantage(torch.zeros(2), off)
    with pytest.raises(TypeError, match="logp"):
        T.tree_ens_policy_loss(torch.zeros(2), None, torch.zeros(1), off)


def test_binding_refuses_a_stream_of_another_device(monkeypatch):
    """Work on it would go to the tensors' device all the same, unordered with it."""
    import torch
    from types import SimpleNamespace

    from paper_1212_2287_amd import _binding as B
    monkeypatch.setattr(torch.cuda, "stream", lambda stream: ("inside", stream))
    here, there = (SimpleNamespace(cuda_stream=7, device=torch.device("cuda", k)) for k in (0, 1))
    assert B._elsewhere(torch.device("cuda", 0), here) == ("inside", here)
    with pytest.raises(TypeError, match="stream"):
        B._elsewhere(torch.device("cuda", 0), there)
