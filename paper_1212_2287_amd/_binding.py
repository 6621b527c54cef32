"""ctypes binding of ``libtreeens.so``: the C ABI of ``include/tree_ens.h`` under the same
names, plus a small ``TreeEnsemble`` owner class. Argument marshalling only -- every step of
scoring runs in the HIP kernels; torch supplies device memory and the current stream.

The library is loaded from this package's directory and never built here: if it is missing the
first call raises ``TreeEnsLibraryMissing`` (build it with ``__graft_entry__.build()``).
"""
from __future__ import annotations

import array
import ctypes
import os
import re
from operator import attrgetter
from typing import Optional

import numpy as np

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "libtreeens.so")
HEADER = os.path.join(os.path.dirname(PKG), "include", "tree_ens.h")

TREE_ENS_OK = 0
TREE_ENS_E_ARG = -1
TREE_ENS_E_MODEL = -2
TREE_ENS_E_SHAPE = -3
TREE_ENS_E_DEVICE = -4
TREE_ENS_E_NOMEM = -5
TREE_ENS_RIGHT_IF_GE = 0
TREE_ENS_RIGHT_IF_GT = 1
(TREE_ENS_PATH_NONE, TREE_ENS_PATH_WALK, TREE_ENS_PATH_UNIFORM, TREE_ENS_PATH_TERMINAL, TREE_ENS_PATH_ROWS,
 TREE_ENS_PATH_CODEGEN) = range(6)
TREE_ENS_CODEGEN = 2  # also compile a kernel specialised for the model (hiprtc)
TREE_ENS_F32, TREE_ENS_BF16, TREE_ENS_F16 = range(3)  # types of logits
TREE_ENS_SEQ_MEAN = 1  # a sequence counts with the mean over its tokens, not the sum
TREE_ENS_CENTER_ONLY = 2  # advantages are not divided by the standard deviation

_dtype_of, _shape_of = attrgetter("dtype"), attrgetter("shape")

_CODE_NAMES = {0: "OK", -1: "E_ARG", -2: "E_MODEL", -3: "E_SHAPE", -4: "E_DEVICE", -5: "E_NOMEM"}


class TreeEnsLibraryMissing(RuntimeError):
    pass


class TreeEnsError(RuntimeError):
    def __init__(self, code: int, where: str, message: str):
        super().__init__(f"{where}: {_CODE_NAMES.get(code, code)} ({code}): {message}")
        self.code = code
        self.message = message


_lib: Optional[ctypes.CDLL] = None


def load_library(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load (once) and return the HIP library; raise if it has not been built."""
    global _lib
    if _lib is not None and path == LIB_PATH:
        return _lib
    # torch ships its own HIP runtime under the same soname (libamdhip64.so.7) as the system
    # one this library links against. Importing torch first makes the loader resolve this
    # library's dependency to the runtime torch already uses, so the process has one HIP
    # runtime and torch's streams and allocations are valid here.
    import torch  # noqa: F401
    if not os.path.exists(path):
        raise TreeEnsLibraryMissing(
            f"{path} is missing: the gfx950 HIP library must be built (__graft_entry__.build())")
    lib = ctypes.CDLL(path)
    P, i32, i64, u32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_uint32
    lib.tree_ens_create.restype = ctypes.c_int
    lib.tree_ens_create.argtypes = [ctypes.POINTER(P), i32, P, P, P, P, P, P, u32]
    lib.tree_ens_create_multi.restype = ctypes.c_int
    lib.tree_ens_create_multi.argtypes = [ctypes.POINTER(P), i32, P, P, P, P, P, P, i32, i32, u32]
    lib.tree_ens_codegen_source.restype = ctypes.c_int
    lib.tree_ens_codegen_source.argtypes = [i32, P, P, P, P, P, P, u32, P, i64, P]
    lib.tree_ens_outputs.restype = ctypes.c_int
    lib.tree_ens_outputs.argtypes = [P, P, P]
    lib.tree_ens_kernel_timing.restype = ctypes.c_int
    lib.tree_ens_kernel_timing.argtypes = [P, i32]
    lib.tree_ens_kernel_time.restype = ctypes.c_int
    lib.tree_ens_kernel_time.argtypes = [P, P, P]
    lib.tree_ens_last_path.restype = ctypes.c_int
    lib.tree_ens_last_path.argtypes = [P, P]
    lib.tree_ens_predict.restype = ctypes.c_int
    lib.tree_ens_predict.argtypes = [P, P, P, i64, i32, P]
    lib.tree_ens_predict_noalloc.restype = ctypes.c_int
    lib.tree_ens_predict_noalloc.argtypes = [P, P, P, i64, i32, P]
    lib.tree_ens_predict_leaves.restype = ctypes.c_int
    lib.tree_ens_predict_leaves.argtypes = [P, P, P, i64, i32, P]
    lib.tree_ens_topk.restype = ctypes.c_int
    lib.tree_ens_feature_usage.restype = ctypes.c_int
    lib.tree_ens_feature_usage.argtypes = [P, P, P, i64, i32, P, P]
    lib.tree_ens_topk.argtypes = [P, P, i64, P, i64, i32, P, P]
    lib.tree_ens_predict_topk.restype = ctypes.c_int
    lib.tree_ens_predict_topk.argtypes = [P, P, P, i64, i32, P, i64, i32, P, P, P]
    lib.tree_ens_info.restype = ctypes.c_int
    lib.tree_ens_info.argtypes = [P, P, P, P, P, P, P]
    f32 = ctypes.c_float
    for name, args in {
            "tree_ens_token_logp": [P, P, i32, i64, i64, i64, P, f32, P, P, P, P, i64],
            "tree_ens_token_logp_workspace": [i32, i64, i64, P],
            "tree_ens_token_logp_backward": [P, P, i32, i64, i64, i64, P, f32, P, P, P, P, P, i64],
            "tree_ens_preference_loss": [P, P, P, P, i64, P, i64, P, P, i64, f32, f32, f32, u32, P, P, P, P, i64],
            "tree_ens_preference_workspace": [i64, i64, i64, P],
            "tree_ens_group_advantage": [P, P, i64, P, i64, f32, u32, P],
            "tree_ens_policy_loss": [P, P, P, P, P, i64, P, i64, P, f32, f32, f32, f32, u32, P, P, P, P, i64],
            "tree_ens_policy_workspace": [i64, i64, P],
            "tree_ens_sample": [P, P, i32, i64, i64, i64, P, f32, i32, f32, f32, P, P, P, P, P, P, P, P, i64],
            "tree_ens_sample_workspace": [i32, i64, i64, P],
            "tree_ens_grad_norm": [P, i64, P, P, P, P, P, i64],
            "tree_ens_grad_norm_workspace": [i64, P],
            "tree_ens_grad_clip": [P, i64, P, P, P, P, f32, f32, P]}.items():
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = ctypes.c_int, args
    lib.tree_ens_destroy.restype = None
    lib.tree_ens_destroy.argtypes = [P]
    lib.tree_ens_last_error.restype = ctypes.c_char_p
    lib.tree_ens_last_error.argtypes = []
    if path == LIB_PATH:
        _lib = lib
    return lib


def header_functions(header: str = HEADER) -> list[str]:
    """Names of the functions ``include/tree_ens.h`` declares."""
    text = open(header).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    return sorted(set(re.findall(r"\b(tree_ens_[a-z_]+)\s*\(", text)))


def tree_ens_last_error() -> str:
    return load_library().tree_ens_last_error().decode()


def _check(rc: int, where: str) -> None:
    if rc != TREE_ENS_OK:
        raise TreeEnsError(rc, where, tree_ens_last_error())


def _arr(a, dtype):
    return np.ascontiguousarray(np.asarray(a), dtype=dtype)


def _model_args(tree_offsets, feature, threshold, left, right, value, n_outputs=1):
    off = _arr(tree_offsets, np.int64)
    fe, th = _arr(feature, np.int32), _arr(threshold, np.float32)
    le, ri, va = _arr(left, np.int32), _arr(right, np.int32), _arr(value, np.float32)
    n_trees = int(off.shape[0]) - 1
    if n_trees < 0:
        raise ValueError("tree_offsets needs n_trees + 1 entries")
    n = int(off[-1]) if n_trees > 0 else 0
    for name, a in (("feature", fe), ("threshold", th), ("left", le), ("right", ri)):
        if a.shape[0] < n:
            raise ValueError(f"{name} has {a.shape[0]} entries; tree_offsets asks for {n}")
    if va.size < n * n_outputs:
        raise ValueError(f"value has {va.size} entries; {n} nodes x {n_outputs} outputs are needed")

    def ptr(a):
        return a.ctypes.data if a.size else None

    # the arrays are returned too: they must outlive the call
    return n_trees, [ptr(a) for a in (off, fe, th, le, ri, va)], (off, fe, th, le, ri, va)


def tree_ens_create(tree_offsets, feature, threshold, left, right, value,
                    flags: int = TREE_ENS_RIGHT_IF_GE) -> ctypes.c_void_p:
    """Validate, pack and upload an ensemble given as flat creation-order arrays (host)."""
    lib = load_library()
    n_trees, ptrs, _keep = _model_args(tree_offsets, feature, threshold, left, right, value)
    h = ctypes.c_void_p()
    rc = lib.tree_ens_create(ctypes.byref(h), n_trees, *ptrs, int(flags))
    _check(rc, "tree_ens_create")
    return h


def tree_ens_create_multi(tree_offsets, feature, threshold, left, right, value, n_outputs: int,
                          n_bags: int = 1, flags: int = TREE_ENS_RIGHT_IF_GE) -> ctypes.c_void_p:
    """tree_ens_create with leaf rows of ``n_outputs`` values (``value`` [n_nodes, n_outputs])
    and ``n_bags`` averaged bags."""
    lib = load_library()
    n_trees, ptrs, _keep = _model_args(tree_offsets, feature, threshold, left, right, value, n_outputs)
    h = ctypes.c_void_p()
    rc = lib.tree_ens_create_multi(ctypes.byref(h), n_trees, *ptrs, int(n_outputs), int(n_bags), int(flags))
    _check(rc, "tree_ens_create_multi")
    return h


def tree_ens_codegen_source(tree_offsets, feature, threshold, left, right, value,
                            flags: int = TREE_ENS_RIGHT_IF_GE) -> str:
    """The HIP source TREE_ENS_CODEGEN compiles for the model (host only)."""
    lib = load_library()
    n_trees, ptrs, _keep = _model_args(tree_offsets, feature, threshold, left, right, value)
    n = ctypes.c_int64()
    _check(lib.tree_ens_codegen_source(n_trees, *ptrs, int(flags), None, 0, ctypes.byref(n)),
           "tree_ens_codegen_source")
    buf = ctypes.create_string_buffer(n.value + 1)
    _check(lib.tree_ens_codegen_source(n_trees, *ptrs, int(flags), buf, n.value + 1, None),
           "tree_ens_codegen_source")
    return buf.value.decode()


def tree_ens_outputs(h) -> tuple[int, int]:
    """(n_outputs, n_bags) of a handle."""
    n_out, n_bags = ctypes.c_int32(), ctypes.c_int32()
    _check(load_library().tree_ens_outputs(h, ctypes.byref(n_out), ctypes.byref(n_bags)), "tree_ens_outputs")
    return n_out.value, n_bags.value


def tree_ens_kernel_timing(h, enable: bool) -> None:
    """Start (a new record) or stop timing the scoring launches of later predicts."""
    _check(load_library().tree_ens_kernel_timing(h, 1 if enable else 0), "tree_ens_kernel_timing")


def tree_ens_kernel_time(h) -> tuple[float, int]:
    """(total milliseconds, launches) of the scoring launches timed since the last start."""
    ms, n = ctypes.c_double(), ctypes.c_int32()
    _check(load_library().tree_ens_kernel_time(h, ctypes.byref(ms), ctypes.byref(n)), "tree_ens_kernel_time")
    return ms.value, n.value


def tree_ens_last_path(h) -> int:
    """Which kernels the handle's last call enqueued (TREE_ENS_PATH_*)."""
    path = ctypes.c_int32()
    _check(load_library().tree_ens_last_path(h, ctypes.byref(path)), "tree_ens_last_path")
    return path.value


def _stream_of(t, stream) -> Optional[int]:
    import torch
    if stream is None:
        # the raw handle of torch's current stream on X's device (cheaper than building a
        # Stream object per call)
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        if raw is not None:
            return raw(t.device.index)
        return torch.cuda.current_stream(t.device).cuda_stream
    return int(getattr(stream, "cuda_stream", stream))


def _check_docs(X):
    import torch
    if not isinstance(X, torch.Tensor) or X.device.type != "cuda":
        raise TypeError("X must be a CUDA (HIP) torch tensor")
    if X.dtype != torch.float32 or X.dim() != 2 or not X.is_contiguous():
        raise TypeError("X must be a contiguous float32 [n_docs, n_features] tensor")


def tree_ens_predict(h, X, scores=None, stream=None, n_outputs=None, _noalloc=False):
    """Scores of the documents ``X`` (device float32 [n_docs, n_features]) as float32 [n_docs]
    (or [n_docs, n_outputs] for a handle with several outputs), enqueued on ``stream``
    (default: torch's current stream for X's device)."""
    import torch
    _check_docs(X)
    n_docs, n_feat = X.shape
    if n_outputs is None:
        n_outputs = tree_ens_outputs(h)[0]
    if scores is None:
        shape = (n_docs,) if n_outputs == 1 else (n_docs, n_outputs)
        scores = torch.empty(shape, dtype=torch.float32, device=X.device)
    elif scores.dtype != torch.float32 or scores.numel() < n_docs * n_outputs or \
            not scores.is_contiguous() or scores.device != X.device:
        raise TypeError("scores must be a contiguous float32 tensor of n_docs * n_outputs entries "
                        "on X's device")
    fn = "tree_ens_predict_noalloc" if _noalloc else "tree_ens_predict"
    rc = getattr(load_library(), fn)(h, _stream_of(X, stream), X.data_ptr() if n_docs else None,
                                     n_docs, n_feat, scores.data_ptr() if n_docs else None)
    _check(rc, fn)
    return scores


def tree_ens_predict_noalloc(h, X, scores, stream=None, n_outputs=None):
    """tree_ens_predict through the allocation-free entry point: ``scores`` must be given (a
    device float32 tensor of n_docs * n_outputs entries); the library allocates nothing."""
    if scores is None:
        raise TypeError("tree_ens_predict_noalloc needs a preallocated scores tensor")
    return tree_ens_predict(h, X, scores, stream, n_outputs, _noalloc=True)


def tree_ens_predict_leaves(h, X, leaf_ids=None, stream=None):
    """Leaf reached per (document, tree), int32 [n_docs, n_trees], tree-local input node ids."""
    import torch
    _check_docs(X)
    n_docs, n_feat = X.shape
    n_trees = tree_ens_info(h)["n_trees"]
    if leaf_ids is None:
        leaf_ids = torch.empty((n_docs, n_trees), dtype=torch.int32, device=X.device)
    elif leaf_ids.dtype != torch.int32 or leaf_ids.numel() < n_docs * n_trees or \
            not leaf_ids.is_contiguous() or leaf_ids.device != X.device:
        raise TypeError("leaf_ids must be a contiguous int32 tensor of n_docs*n_trees entries")
    rc = load_library().tree_ens_predict_leaves(h, _stream_of(X, stream), X.data_ptr() if n_docs else None,
                                                n_docs, n_feat,
                                                leaf_ids.data_ptr() if n_docs * n_trees else None)
    _check(rc, "tree_ens_predict_leaves")
    return leaf_ids


def tree_ens_feature_usage(h, X, counts=None, masks=None, want_masks: bool = True, stream=None):
    """Features examined per document over all trees: (counts int32 [n_docs], masks int32
    [n_docs, (n_features + 31) // 32] holding the uint32 bit patterns, or None when
    ``want_masks`` is false and no ``masks`` tensor is given)."""
    import torch
    _check_docs(X)
    n_docs, n_feat = X.shape
    words = (n_feat + 31) // 32
    if counts is None:
        counts = torch.empty(n_docs, dtype=torch.int32, device=X.device)
    elif counts.dtype != torch.int32 or counts.numel() < n_docs or not counts.is_contiguous() \
            or counts.device != X.device:
        raise TypeError("counts must be a contiguous int32 tensor of n_docs entries on X's device")
    if masks is None and want_masks:
        masks = torch.empty((n_docs, words), dtype=torch.int32, device=X.device)
    if masks is not None and (masks.dtype != torch.int32 or masks.numel() < n_docs * words or
                              not masks.is_contiguous() or masks.device != X.device):
        raise TypeError("masks must be a contiguous int32 tensor of n_docs*words entries on X's device")
    rc = load_library().tree_ens_feature_usage(
        h, _stream_of(X, stream), X.data_ptr() if n_docs else None, n_docs, n_feat,
        counts.data_ptr() if n_docs else None,
        masks.data_ptr() if masks is not None and n_docs else None)
    _check(rc, "tree_ens_feature_usage")
    return counts, masks


def _topk_outputs(device, n_groups, k, top_idx, top_scores):
    import torch
    if top_idx is None:
        top_idx = torch.empty((n_groups, k), dtype=torch.int32, device=device)
    elif top_idx.dtype != torch.int32 or top_idx.numel() < n_groups * k or not top_idx.is_contiguous() \
            or top_idx.device != device:
        raise TypeError("top_idx must be a contiguous int32 tensor of n_groups*k entries on the device")
    if top_scores is None:
        top_scores = torch.empty((n_groups, k), dtype=torch.float32, device=device)
    elif top_scores.dtype != torch.float32 or top_scores.numel() < n_groups * k or \
            not top_scores.is_contiguous() or top_scores.device != device:
        raise TypeError("top_scores must be a contiguous float32 tensor of n_groups*k entries")
    return top_idx, top_scores


def _check_offsets(group_offsets, device):
    import torch
    if not isinstance(group_offsets, torch.Tensor) or group_offsets.dtype != torch.int64 or \
            group_offsets.dim() != 1 or not group_offsets.is_contiguous() or \
            group_offsets.device != device or group_offsets.numel() < 1:
        raise TypeError("group_offsets must be a contiguous int64 [n_groups + 1] tensor on the device")
    return group_offsets.numel() - 1


def tree_ens_topk(scores, group_offsets, k: int, top_idx=None, top_scores=None, stream=None):
    """Per-group top-k of device float32 ``scores`` over the groups of ``group_offsets`` (device
    int64 [n_groups + 1]): (top_idx int32 [n_groups, k], top_scores float32 [n_groups, k])."""
    import torch
    if not isinstance(scores, torch.Tensor) or scores.device.type != "cuda" or \
            scores.dtype != torch.float32 or scores.dim() != 1 or not scores.is_contiguous():
        raise TypeError("scores must be a contiguous float32 CUDA (HIP) vector")
    n_groups = _check_offsets(group_offsets, scores.device)
    top_idx, top_scores = _topk_outputs(scores.device, n_groups, k, top_idx, top_scores)
    rc = load_library().tree_ens_topk(_stream_of(scores, stream), scores.data_ptr() if scores.numel() else None,
                                      scores.numel(), group_offsets.data_ptr(), n_groups, int(k),
                                      top_idx.data_ptr() if n_groups else None,
                                      top_scores.data_ptr() if n_groups else None)
    _check(rc, "tree_ens_topk")
    return top_idx, top_scores


def tree_ens_predict_topk(h, X, group_offsets, k: int, scores=None, top_idx=None, top_scores=None,
                          stream=None):
    """Scores of ``X`` and their per-group top-k in one call: (scores, top_idx, top_scores)."""
    import torch
    _check_docs(X)
    n_docs, n_feat = X.shape
    if scores is None:
        scores = torch.empty(n_docs, dtype=torch.float32, device=X.device)
    elif scores.dtype != torch.float32 or scores.numel() < n_docs or not scores.is_contiguous() \
            or scores.device != X.device:
        raise TypeError("scores must be a contiguous float32 tensor of n_docs entries on X's device")
    n_groups = _check_offsets(group_offsets, X.device)
    top_idx, top_scores = _topk_outputs(X.device, n_groups, k, top_idx, top_scores)
    rc = load_library().tree_ens_predict_topk(
        h, _stream_of(X, stream), X.data_ptr() if n_docs else None, n_docs, n_feat,
        group_offsets.data_ptr(), n_groups, int(k), scores.data_ptr() if n_docs else None,
        top_idx.data_ptr() if n_groups else None, top_scores.data_ptr() if n_groups else None)
    _check(rc, "tree_ens_predict_topk")
    return scores, top_idx, top_scores


# ----------------------------------------------------------------------------------------------
# learning from scores
#
# No call records an autograd graph, whether its inputs require gradients or not: what it returns has none, and
# gradients are handed on by the caller (logits.backward(grad_logits) where torch made the logits).
# ----------------------------------------------------------------------------------------------
def _vector(name, t, dtypes, n, device):
    """Check a contiguous device vector of n entries (any number if n is None)."""
    import torch
    if isinstance(t, torch.Tensor) and t.dtype in dtypes and t.dim() == 1 and t.is_contiguous() and \
            (t.device == device if device is not None else t.is_cuda):
        if n is None or t.numel() == n:
            return t
        raise TypeError(f"{name} must have {n} entries, not {t.numel()}")
    raise TypeError(f"{name} must be a contiguous {str(dtypes[0])[6:]} vector on the device")


def _ptr(t):
    return t.data_ptr() or None if t is not None else None


def _elsewhere(device, stream):
    """A context in which ``stream`` is torch's current stream on ``device``, or None where it is already: the call
    then runs inside it, so that memory it allocates belongs to the stream its work runs on."""
    import torch
    if stream is None:
        return None if torch.cuda.current_device() == device.index else torch.cuda.device(device)
    if not hasattr(stream, "cuda_stream"):
        stream = torch.cuda.ExternalStream(int(stream), device)
    elif stream.device != device:
        raise TypeError(f"stream must be on the tensors' device {device}, not on {stream.device}")
    return torch.cuda.stream(stream)


def _workspace(lib, device, fn, *sizes):
    """(tensor or None, pointer, bytes) that the function of these sizes needs."""
    import torch
    need = ctypes.c_int64()
    _check(getattr(lib, fn)(*sizes, ctypes.byref(need)), fn)
    if not need.value:
        return None, None, 0
    t = torch.empty(need.value, dtype=torch.uint8, device=device)
    return t, t.data_ptr(), need.value


def _stream_on(device):
    """torch's current stream on a device, as tree_ens_predict takes it."""
    import torch
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return raw(device.index) if raw is not None else torch.cuda.current_stream(device).cuda_stream


def _dtype_codes():
    import torch
    return {torch.float32: TREE_ENS_F32, torch.bfloat16: TREE_ENS_BF16, torch.float16: TREE_ENS_F16}


def _check_logits(logits, targets, name="targets", dtype=None):
    """(dtype code, n_tokens, n_vocab, row stride) of device logits [n_tokens, n_vocab] and a vector over their rows."""
    import torch
    codes = _dtype_codes()
    if not isinstance(logits, torch.Tensor) or not logits.is_cuda or logits.dtype not in codes or \
            logits.dim() != 2 or (logits.shape[1] > 1 and logits.stride(1) != 1):
        raise TypeError("logits must be a CUDA (HIP) float32, bfloat16 or float16 [n_tokens, n_vocab] tensor with "
                        "contiguous rows")
    n, v = logits.shape
    _vector(name, targets, (dtype or torch.int64,), n, logits.device)
    return codes[logits.dtype], n, v, logits.stride(0) if n > 1 else v


def _check_stats(stats, n, device):
    import torch
    if not isinstance(stats, torch.Tensor) or stats.dtype != torch.float32 or stats.shape != (n, 2) or \
            not stats.is_contiguous() or stats.device != device:
        raise TypeError("stats must be a contiguous float32 [n_tokens, 2] tensor on the logits' device")


def tree_ens_token_logp(logits, targets, scale: float = 1.0, want_entropy: bool = False, logp=None, entropy=None,
                        stats=None, stream=None):
    """Log-probabilities of ``targets`` (device int64 [n_tokens]; outside [0, n_vocab): not counted) under
    softmax(scale * logits): (logp float32 [n_tokens], entropy float32 [n_tokens] or None, stats float32
    [n_tokens, 2] for the gradient). Rows of ``logits`` may lie any stride apart. No autograd graph is recorded:
    tree_ens_token_logp_backward gives the gradient."""
    import torch
    code, n, v, stride = _check_logits(logits, targets)
    f32, dev = torch.float32, logits.device
    elsewhere = _elsewhere(dev, stream)
    if elsewhere is not None:
        with elsewhere:
            return tree_ens_token_logp(logits, targets, scale, want_entropy, logp, entropy, stats)
    if logp is None:
        logp = torch.empty(n, dtype=f32, device=dev)
    else:
        _vector("logp", logp, (f32,), n, dev)
    if entropy is not None:
        _vector("entropy", entropy, (f32,), n, dev)
    elif want_entropy:
        entropy = torch.empty(n, dtype=f32, device=dev)
    if stats is None:
        stats = torch.empty((n, 2), dtype=f32, device=dev)
    else:
        _check_stats(stats, n, dev)
    lib = load_library()
    _keep, work, size = _workspace(lib, dev, "tree_ens_token_logp_workspace", code, n, v)
    _check(lib.tree_ens_token_logp(_stream_on(dev), _ptr(logits), code, n, v, stride, _ptr(targets), float(scale),
           _ptr(logp), _ptr(entropy), _ptr(stats), work, size), "tree_ens_token_logp")
    return logp, entropy, stats


def tree_ens_token_logp_backward(logits, targets, stats, grad_logp, scale: float = 1.0, entropy=None, grad_entropy=None,
                                 grad_logits=None, stream=None):
    """The gradient of sum(grad_logp * logp + grad_entropy * entropy) with respect to ``logits``, in their type
    (``entropy`` as the forward gave it; both or neither). ``grad_logits`` may be ``logits`` itself.
    ``logits.backward(grad_logits)`` hands it on where torch's autograd made the logits."""
    import torch
    code, n, v, stride = _check_logits(logits, targets)
    f32, dev = torch.float32, logits.device
    _check_stats(stats, n, dev)
    _vector("grad_logp", grad_logp, (f32,), n, dev)
    if (entropy is None) != (grad_entropy is None):
        raise TypeError("entropy and grad_entropy are given together")
    if entropy is not None:
        _vector("entropy", entropy, (f32,), n, dev)
        _vector("grad_entropy", grad_entropy, (f32,), n, dev)
    elsewhere = _elsewhere(dev, stream)
    if elsewhere is not None:
        with elsewhere:
            return tree_ens_token_logp_backward(logits, targets, stats, grad_logp, scale, entropy, grad_entropy, grad_logits)
    if grad_logits is None:
        grad_logits = torch.empty((n, v), dtype=logits.dtype, device=dev)
    elif not isinstance(grad_logits, torch.Tensor) or grad_logits.dtype != logits.dtype or \
            grad_logits.shape != logits.shape or (v > 1 and grad_logits.stride(1) != 1) or grad_logits.device != dev:
        raise TypeError("grad_logits must be a tensor of the logits' type, shape and device with contiguous rows")
    _check(load_library().tree_ens_token_logp_backward(_stream_on(dev), _ptr(logits), code, n, v, stride,
           _ptr(targets), float(scale), _ptr(stats), _ptr(grad_logp), _ptr(entropy), _ptr(grad_entropy), _ptr(grad_logits),
           grad_logits.stride(0) if n > 1 else v), "tree_ens_token_logp_backward")
    return grad_logits


def _check_tokens(logp, seq_offsets, mask, **others):
    """(n_tokens, n_seqs) of packed sequences; `others` are float vectors over the tokens, or None."""
    import torch
    f32 = (torch.float32,)
    _vector("logp", logp, f32, None, None)
    n, dev = logp.shape[0], logp.device
    for name, t in others.items():
        if t is not None:
            _vector(name, t, f32, n, dev)
    if mask is not None:
        _vector("mask", mask, (torch.bool, torch.uint8), n, dev)
    _vector("seq_offsets", seq_offsets, (torch.int64,), None, dev)
    if seq_offsets.shape[0] < 1:
        raise TypeError("seq_offsets must have n_seqs + 1 entries")
    return n, seq_offsets.shape[0] - 1


def _float_out(name, t, n, device):
    """A float vector of n entries: the caller's, or a new one."""
    import torch
    if t is None:
        return torch.empty(n, dtype=torch.float32, device=device)
    return _vector(name, t, (torch.float32,), n, device)


def tree_ens_preference_loss(logp, seq_offsets, scores, group_offsets, ref_logp=None, mask=None, beta: float = 0.1,
                             smoothing: float = 0.0, grad_scale: float = 1.0, flags: int = 0, want_grad: bool = True,
                             loss=None, margins=None, grad_logp=None, stream=None):
    """Pairwise preference loss of each group's sequences, in the order of their ``scores``, on log ratios to a
    reference model: (loss float32 [n_groups], margins float32 [n_seqs], gradient of grad_scale * loss.sum() with
    respect to ``logp``, or None without ``want_grad``). No autograd graph is recorded."""
    import torch
    n, n_seqs = _check_tokens(logp, seq_offsets, mask, ref_logp=ref_logp, grad_logp=grad_logp)
    dev = logp.device
    _vector("scores", scores, (torch.float32,), n_seqs, dev)
    n_groups = _check_offsets(group_offsets, dev)
    elsewhere = _elsewhere(dev, stream)
    if elsewhere is not None:
        with elsewhere:
            return tree_ens_preference_loss(logp, seq_offsets, scores, group_offsets, ref_logp, mask, beta, smoothing,
                                            grad_scale, flags, want_grad, loss, margins, grad_logp)
    loss = _float_out("loss", loss, n_groups, dev)
    margins = _float_out("margins", margins, n_seqs, dev)
    if grad_logp is None and want_grad:
        grad_logp = torch.empty(n, dtype=torch.float32, device=dev)
    lib = load_library()
    _keep, work, size = _workspace(lib, dev, "tree_ens_preference_workspace", n, n_seqs, n_groups)
    _check(lib.tree_ens_preference_loss(_stream_on(dev), _ptr(logp), _ptr(ref_logp), _ptr(mask), n,
           seq_offsets.data_ptr(), n_seqs, _ptr(scores), group_offsets.data_ptr(), n_groups, float(beta), float(smoothing),
           float(grad_scale), int(flags), _ptr(loss), _ptr(margins), _ptr(grad_logp), work, size),
           "tree_ens_preference_loss")
    return loss, margins, grad_logp


def tree_ens_group_advantage(scores, group_offsets, eps: float = 1e-6, flags: int = 0, advantages=None, stream=None):
    """Scores relative to their group, (s - mean) / (std + eps): float32 [n_docs]."""
    import torch
    _vector("scores", scores, (torch.float32,), None, None)
    n, dev = scores.shape[0], scores.device
    n_groups = _check_offsets(group_offsets, dev)
    elsewhere = _elsewhere(dev, stream)
    if elsewhere is not None:
        with elsewhere:
            return tree_ens_group_advantage(scores, group_offsets, eps, flags, advantages)
    advantages = _float_out("advantages", advantages, n, dev)
    _check(load_library().tree_ens_group_advantage(_stream_on(dev), _ptr(scores), n, group_offsets.data_ptr(),
           n_groups, float(eps), int(flags), _ptr(advantages)), "tree_ens_group_advantage")
    return advantages


def tree_ens_policy_loss(logp, old_logp, advantages, seq_offsets, ref_logp=None, mask=None, clip_low: float = 0.2,
                         clip_high: float = 0.2, kl_coef: float = 0.0, grad_scale: float = 1.0, flags: int = 0,
                         want_grad: bool = True, loss=None, kl=None, grad_logp=None, stream=None):
    """Clipped policy loss of each sequence with kl_coef times its KL estimate to a reference model: (loss float32
    [n_seqs], kl float32 [n_seqs] or None without ``ref_logp``, gradient of grad_scale * loss.sum() with respect to
    ``logp``, or None without ``want_grad``). ``old_logp`` None: the tokens were sampled by this very policy.
    No autograd graph is recorded."""
    import torch
    n, n_seqs = _check_tokens(logp, seq_offsets, mask, old_logp=old_logp, ref_logp=ref_logp, grad_logp=grad_logp)
    dev = logp.device
    _vector("advantages", advantages, (torch.float32,), n_seqs, dev)
    elsewhere = _elsewhere(dev, stream)
    if elsewhere is not None:
        with elsewhere:
            return tree_ens_policy_loss(logp, old_logp, advantages, seq_offsets, ref_logp, mask, clip_low, clip_high,
                                        kl_coef, grad_scale, flags, want_grad, loss, kl, grad_logp)
    loss = _float_out("loss", loss, n_seqs, dev)
    if kl is not None or ref_logp is not None:
        kl = _float_out("kl", kl, n_seqs, dev)
    if grad_logp is None and want_grad:
        grad_logp = torch.empty(n, dtype=torch.float32, device=dev)
    lib = load_library()
    _keep, work, size = _workspace(lib, dev, "tree_ens_policy_workspace", n, n_seqs)
    _check(lib.tree_ens_policy_loss(_stream_on(dev), _ptr(logp), _ptr(old_logp), _ptr(ref_logp), _ptr(mask), n,
           seq_offsets.data_ptr(), n_seqs, _ptr(advantages), float(clip_low), float(clip_high), float(kl_coef),
           float(grad_scale), int(flags), _ptr(loss), _ptr(kl), _ptr(grad_logp), work, size), "tree_ens_policy_loss")
    return loss, kl, grad_logp


def _row_parameter(name, value, dtype, n, device):
    """(number, device vector or None) of a parameter that is one number or a vector over the rows."""
    import torch
    if isinstance(value, torch.Tensor):
        return 1, _vector(name, value, (dtype,), n, device)
    return value, None


def tree_ens_sample(logits, uniform, scale=1.0, top_k=0, top_p=1.0, min_p=0.0, want_logp: bool = True, tokens=None, logp=None,
                    log_kept=None, stream=None):
    """One token of every row of ``logits`` (as for tree_ens_token_logp) under softmax(scale * logits) cut down by ``top_k``
    (0: off), ``min_p`` (0: off) and ``top_p`` (1: off), from the random numbers ``uniform`` (device float64 [n_tokens] in
    [0, 1)): (tokens int64 [n_tokens], logp float32 [n_tokens] over the whole vocabulary, as tree_ens_token_logp gives it,
    log_kept float32 [n_tokens], the logarithm of the share of the probability that is kept; both None without
    ``want_logp``). ``scale``, ``top_p`` and ``min_p`` may be device float32 vectors over the rows, ``top_k`` an int32 one."""
    import torch
    f32 = torch.float32
    code, n, v, stride = _check_logits(logits, uniform, "uniform", torch.float64)
    dev = logits.device
    scale_, row_scale = _row_parameter("scale", scale, f32, n, dev)
    top_k_, row_top_k = _row_parameter("top_k", top_k, torch.int32, n, dev)
    top_p_, row_top_p = _row_parameter("top_p", top_p, f32, n, dev)
    min_p_, row_min_p = _row_parameter("min_p", min_p, f32, n, dev)
    elsewhere = _elsewhere(dev, stream)
    if elsewhere is not None:
        with elsewhere:
            return tree_ens_sample(logits, uniform, scale, top_k, top_p, min_p, want_logp, tokens, logp, log_kept)
    if tokens is None:
        tokens = torch.empty(n, dtype=torch.int64, device=dev)
    else:
        _vector("tokens", tokens, (torch.int64,), n, dev)
    if logp is not None or want_logp:
        logp = _float_out("logp", logp, n, dev)
    if log_kept is not None or want_logp:
        log_kept = _float_out("log_kept", log_kept, n, dev)
    lib = load_library()
    _keep, work, size = _workspace(lib, dev, "tree_ens_sample_workspace", code, n, v)
    _check(lib.tree_ens_sample(_stream_on(dev), _ptr(logits), code, n, v, stride, _ptr(uniform), float(scale_),
           max(-1, min(int(top_k_), 2**31 - 1)), float(top_p_), float(min_p_), _ptr(row_scale), _ptr(row_top_k), _ptr(row_top_p),
           _ptr(row_min_p), _ptr(tokens), _ptr(logp), _ptr(log_kept), work, size), "tree_ens_sample")
    return tokens, logp, log_kept


def _dense(t) -> bool:
    """Whether a tensor's elements lie one behind the other, in whatever order of its dimensions."""
    if t.is_contiguous():
        return True
    at = 1
    for stride, size in sorted((st, sz) for st, sz in zip(t.stride(), t.shape) if sz != 1):
        if stride != at:
            return False
        at *= size
    return True


def _check_grads(grads, name="grads"):
    """(device, tensors, their addresses, counts and dtype codes in arrays) of a sequence of dense device tensors. One
    reading of all tensors for each of their properties costs a third of a loop over them."""
    import torch
    grads = list(grads)
    if not grads or not all(issubclass(kind, torch.Tensor) for kind in set(map(type, grads))):
        raise TypeError(f"{name} must be a sequence of one tensor or more")
    Tensor, codes = torch.Tensor, _dtype_codes()
    dtypes = list(map(_dtype_of, grads))
    kinds = set(dtypes)
    if not kinds <= codes.keys() or not (all(map(Tensor.is_contiguous, grads)) or all(map(_dense, grads))):
        raise TypeError(f"{name} must be float32, bfloat16 or float16 tensors without gaps between their elements")
    if not grads[0].is_cuda or len(set(map(Tensor.get_device, grads))) != 1:
        raise TypeError(f"{name} must be CUDA (HIP) tensors of one device")
    kinds = array.array("i", map(codes.__getitem__, dtypes) if len(kinds) > 1 else [codes[dtypes[0]]] * len(grads))
    return grads[0].device, grads, array.array("q", map(Tensor.data_ptr, grads)), array.array("q", map(Tensor.numel, grads)), kinds


def _address(values):
    return values.buffer_info()[0]


def tree_ens_grad_norm(grads, norm=None, stream=None):
    """The 2-norm of the elements of all tensors of ``grads`` together, one or more of them, such as the ``p.grad`` of all
    parameters that have one: a float32 scalar on their device (``norm``, if given). Types may be mixed; tensors are dense, in
    any order of their dimensions."""
    import torch
    dev, grads, ptrs, counts, codes = _check_grads(grads)
    elsewhere = _elsewhere(dev, stream)
    if elsewhere is not None:
        with elsewhere:
            return tree_ens_grad_norm(grads, norm)
    if norm is None:
        norm = torch.empty((), dtype=torch.float32, device=dev)
    else:
        _check_norm(norm, dev)
    lib = load_library()
    _keep, work, size = _workspace(lib, dev, "tree_ens_grad_norm_workspace", len(grads))
    _check(lib.tree_ens_grad_norm(_stream_on(dev), len(grads), _address(ptrs), _address(counts), _address(codes),
           norm.data_ptr(), work, size), "tree_ens_grad_norm")
    return norm


def _check_norm(norm, device):
    import torch
    if not isinstance(norm, torch.Tensor) or norm.dtype != torch.float32 or norm.numel() != 1 or norm.device != device:
        raise TypeError("norm must be a float32 tensor of one element on the gradients' device")


def tree_ens_grad_clip(grads, norm, max_norm: float, eps: float = 1e-6, out=None, stream=None):
    """``grads`` times min(1, max_norm / (norm + eps)), each rounded once to its type, in place or into the tensors of
    ``out`` (of the same shapes, strides and types; they may be some of the same tensors): the tensors written. ``norm`` as
    tree_ens_grad_norm gives it, or over all processes' shards."""
    dev, grads, ptrs, counts, codes = _check_grads(grads)
    _check_norm(norm, dev)
    to = ptrs
    if out is None:
        out = grads
    else:
        out_dev, out, to, _, out_codes = _check_grads(out, "out")
        if out_dev != dev or out_codes != codes or list(map(_shape_of, out)) != list(map(_shape_of, grads)) or \
                any(a.stride() != b.stride() for a, b in zip(out, grads) if not (a.is_contiguous() and b.is_contiguous())):
            raise TypeError("out must hold tensors of the gradients' shapes, strides, types and device")
    elsewhere = _elsewhere(dev, stream)
    if elsewhere is not None:
        with elsewhere:
            return tree_ens_grad_clip(grads, norm, max_norm, eps, out)
    _check(load_library().tree_ens_grad_clip(_stream_on(dev), len(grads), _address(ptrs), _address(counts), _address(codes),
           norm.data_ptr(), float(max_norm), float(eps), _address(to)), "tree_ens_grad_clip")
    return out


def tree_ens_info(h) -> dict:
    lib = load_library()
    nt, mf, md, nt2, dpb = (ctypes.c_int32() for _ in range(5))
    pb = ctypes.c_int64()
    rc = lib.tree_ens_info(h, ctypes.byref(nt), ctypes.byref(mf), ctypes.byref(md), ctypes.byref(pb),
                           ctypes.byref(nt2), ctypes.byref(dpb))
    _check(rc, "tree_ens_info")
    return {"n_trees": nt.value, "min_features": mf.value, "max_depth": md.value,
            "packed_bytes": pb.value, "n_tiles": nt2.value, "docs_per_block": dpb.value}


def tree_ens_destroy(h) -> None:
    if h is not None:
        load_library().tree_ens_destroy(h)


class TreeEnsemble:
    """Owner of a packed model on the current device.

    ``TreeEnsemble.from_arrays(tree_offsets, feature, threshold, left, right, value, flags,
    n_outputs, n_bags)`` or ``TreeEnsemble.from_ensemble(ens, flags, leaf_values, n_bags)`` for
    any object with those attributes; ``TreeEnsemble(handle)`` adopts a handle from the
    module-level create functions. ``n_outputs`` and ``n_bags`` are read back from the handle;
    ``flags`` may include ``TREE_ENS_CODEGEN``."""

    def __init__(self, handle):
        self._h = handle
        self.n_outputs, self.n_bags = tree_ens_outputs(handle)

    @classmethod
    def from_arrays(cls, tree_offsets, feature, threshold, left, right, value,
                    flags: int = TREE_ENS_RIGHT_IF_GE, n_outputs: int = 1, n_bags: int = 1) -> "TreeEnsemble":
        if n_outputs == 1 and n_bags == 1:
            return cls(tree_ens_create(tree_offsets, feature, threshold, left, right, value, flags))
        return cls(tree_ens_create_multi(tree_offsets, feature, threshold, left, right, value,
                                         n_outputs, n_bags, flags))

    @classmethod
    def from_ensemble(cls, ens, flags: int = TREE_ENS_RIGHT_IF_GE, leaf_values=None,
                      n_bags: int = 1) -> "TreeEnsemble":
        """``leaf_values`` [n_nodes, n_outputs] replaces ``ens.value`` (vector-valued leaves)."""
        value, n_out = ens.value, 1
        if leaf_values is not None:
            value = np.ascontiguousarray(leaf_values, dtype=np.float32)
            if value.ndim != 2 or value.shape[0] != ens.n_nodes:
                raise ValueError("leaf_values must be [n_nodes, n_outputs]")
            n_out = value.shape[1]
        return cls.from_arrays(ens.tree_offsets, ens.feature, ens.threshold, ens.left, ens.right,
                               value, flags, n_out, n_bags)

    @property
    def handle(self):
        if self._h is None:
            raise ValueError("model was destroyed")
        return self._h

    def predict(self, X, out=None, stream=None):
        return tree_ens_predict(self.handle, X, out, stream, self.n_outputs)

    def predict_noalloc(self, X, out, stream=None):
        return tree_ens_predict_noalloc(self.handle, X, out, stream, self.n_outputs)

    def predict_leaves(self, X, out=None, stream=None):
        return tree_ens_predict_leaves(self.handle, X, out, stream)

    def feature_usage(self, X, want_masks: bool = True, stream=None):
        return tree_ens_feature_usage(self.handle, X, want_masks=want_masks, stream=stream)

    def predict_topk(self, X, group_offsets, k: int, stream=None):
        """(scores, top_idx, top_scores): scores of X and each query group's k best documents."""
        return tree_ens_predict_topk(self.handle, X, group_offsets, k, stream=stream)

    def info(self) -> dict:
        return tree_ens_info(self.handle)

    def kernel_timing(self, enable: bool) -> None:
        tree_ens_kernel_timing(self.handle, enable)

    def kernel_time(self) -> tuple[float, int]:
        return tree_ens_kernel_time(self.handle)

    def last_path(self) -> int:
        return tree_ens_last_path(self.handle)

    def close(self) -> None:
        if self._h is not None:
            tree_ens_destroy(self._h)
            self._h = None

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
