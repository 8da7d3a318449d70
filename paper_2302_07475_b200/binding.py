"""ctypes binding of libs3gd.so: same names as the C ABI, argument marshalling only.

Every step of the path runs in the CUDA kernels of the library; nothing here
computes.  torch is used for device buffers and the current stream.  If the
library is missing or a tensor is not a contiguous CUDA tensor of the right
dtype the call raises -- there is no CPU fallback.
"""
from __future__ import annotations

import array
import ctypes
import operator
import os
from itertools import chain, repeat
from typing import Optional

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
# S3GD_LIBRARY names another build of the same library (same C ABI) to load instead of the in-tree one
LIB_PATH = os.environ.get("S3GD_LIBRARY") or os.path.join(_PKG, "libs3gd.so")

S3GD_OK = 0
STATUS_NAMES = {
    0: "S3GD_OK", 1: "S3GD_ERR_INVALID_ARG", 2: "S3GD_ERR_WORKSPACE", 3: "S3GD_ERR_CUDA",
    4: "S3GD_ERR_INDEX_RANGE", 5: "S3GD_ERR_INTERNAL", 6: "S3GD_ERR_TOO_LARGE",
}

EXPORTS = ("s3gd_status_string", "s3gd_workspace_bytes", "s3gd_topk_sign", "s3gd_majority_vote",
           "s3gd_apply", "s3gd_step", "s3gd_device_status", "s3gd_profile_begin", "s3gd_profile_end",
           "s3gd_noalloc_max_d", "s3gd_majority_vote_noalloc", "s3gd_step_ex", "s3gd_apply_momentum",
           "s3gd_randk_sign", "s3gd_step_randk", "s3gd_profile_begin_filter", "s3gd_last_device_status",
           "s3gd_debug_topk_sign", "s3gd_debug_step", "s3gd_vote_apply", "s3gd_vote_counts", "s3gd_encode_vote2",
           "s3gd_apply_vote2", "s3gd_sparse_workspace_bytes", "s3gd_encode_vote_sparse", "s3gd_apply_vote_sparse",
           "s3gd_profile_begin_filter_every", "s3gd_orthogonalise_workspace_bytes", "s3gd_orthogonalise", "s3gd_step_ortho",
           "s3gd_embed", "s3gd_embed_grad_workspace_bytes", "s3gd_embed_grad", "s3gd_layer_norm",
           "s3gd_layer_norm_grad_workspace_bytes", "s3gd_layer_norm_grad", "s3gd_clip_workspace_bytes", "s3gd_grad_norm", "s3gd_clip")


class S3gdError(RuntimeError):
    def __init__(self, call: str, code: int):
        super().__init__(f"{call} returned {STATUS_NAMES.get(code, code)}")
        self.code = code


class Matrix(ctypes.Structure):
    """s3gd_matrix of the C ABI."""

    _fields_ = [("data", ctypes.c_void_p), ("dtype", ctypes.c_int), ("row_stride", ctypes.c_int64), ("batch_stride", ctypes.c_int64)]


_lib = None


def load(path: Optional[str] = None) -> ctypes.CDLL:
    """Load the shared library (once) and declare the argument types of every export."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or LIB_PATH
    if not os.path.exists(p):
        raise FileNotFoundError(
            f"{p} not found: build it with `python -m paper_2302_07475_b200.build` (needs nvcc); "
            "there is no fallback implementation")
    lib = ctypes.CDLL(p)
    vp, u64, u32p, sz = ctypes.c_void_p, ctypes.c_uint64, ctypes.c_void_p, ctypes.c_size_t
    lib.s3gd_status_string.restype = ctypes.c_char_p
    lib.s3gd_status_string.argtypes = [ctypes.c_int]
    lib.s3gd_workspace_bytes.restype = sz
    lib.s3gd_workspace_bytes.argtypes = [ctypes.c_int, u64, u64]
    lib.s3gd_topk_sign.restype = ctypes.c_int
    lib.s3gd_topk_sign.argtypes = [vp, ctypes.c_int, u64, u64, u32p, u32p, vp, sz, vp]
    lib.s3gd_majority_vote.restype = ctypes.c_int
    lib.s3gd_majority_vote.argtypes = [u32p, u32p, ctypes.c_int, u64, u64, vp, vp, sz, vp]
    lib.s3gd_apply.restype = ctypes.c_int
    lib.s3gd_apply.argtypes = [vp, vp, u64, ctypes.c_float, vp]
    lib.s3gd_step.restype = ctypes.c_int
    lib.s3gd_step.argtypes = [vp, vp, ctypes.c_int, u64, u64, ctypes.c_float, u32p, u32p, vp, vp, sz, vp]
    lib.s3gd_device_status.restype = ctypes.c_int
    lib.s3gd_device_status.argtypes = [vp, vp, ctypes.c_void_p]
    lib.s3gd_profile_begin.restype = ctypes.c_int
    lib.s3gd_profile_begin.argtypes = [ctypes.c_int]
    lib.s3gd_profile_end.restype = ctypes.c_int
    lib.s3gd_profile_end.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]
    lib.s3gd_noalloc_max_d.restype = ctypes.c_uint64
    lib.s3gd_noalloc_max_d.argtypes = []
    lib.s3gd_majority_vote_noalloc.restype = ctypes.c_int
    lib.s3gd_majority_vote_noalloc.argtypes = [u32p, u32p, ctypes.c_int, u64, u64, vp, vp, vp]
    lib.s3gd_step_ex.restype = ctypes.c_int
    lib.s3gd_step_ex.argtypes = [vp, vp, vp, ctypes.c_float, vp, ctypes.c_float, ctypes.c_int, u64, u64, ctypes.c_float,
                                 u32p, u32p, vp, vp, sz, vp]
    lib.s3gd_apply_momentum.restype = ctypes.c_int
    lib.s3gd_apply_momentum.argtypes = [vp, vp, vp, u64, ctypes.c_float, ctypes.c_float, vp]
    lib.s3gd_profile_begin_filter.restype = ctypes.c_int
    lib.s3gd_profile_begin_filter.argtypes = [ctypes.c_int]
    lib.s3gd_profile_begin_filter_every.restype = ctypes.c_int
    lib.s3gd_profile_begin_filter_every.argtypes = [ctypes.c_int, ctypes.c_int]
    u32 = ctypes.c_uint32
    lib.s3gd_randk_sign.restype = ctypes.c_int
    lib.s3gd_randk_sign.argtypes = [vp, ctypes.c_int, u64, u64, u32, u32, u32p, u32p, vp, sz, vp]
    lib.s3gd_step_randk.restype = ctypes.c_int
    lib.s3gd_step_randk.argtypes = [vp, vp, ctypes.c_int, u64, u64, ctypes.c_float, u32, u32, u32p, u32p, vp, vp, sz, vp]
    lib.s3gd_last_device_status.restype = ctypes.c_int
    lib.s3gd_last_device_status.argtypes = [vp, vp]
    lib.s3gd_debug_topk_sign.restype = ctypes.c_int
    lib.s3gd_debug_topk_sign.argtypes = lib.s3gd_topk_sign.argtypes + [u32]
    lib.s3gd_debug_step.restype = ctypes.c_int
    lib.s3gd_debug_step.argtypes = lib.s3gd_step.argtypes + [u32, u32]
    lib.s3gd_vote_apply.restype = ctypes.c_int
    lib.s3gd_vote_apply.argtypes = [vp, u32p, ctypes.c_int, u64, ctypes.c_int, u64, u64, ctypes.c_float, vp, vp, sz, vp]
    lib.s3gd_vote_counts.restype = ctypes.c_int
    lib.s3gd_vote_counts.argtypes = [u32p, u32p, ctypes.c_int, u64, u64, u64, vp, ctypes.c_int, vp, vp]
    lib.s3gd_encode_vote2.restype = ctypes.c_int
    lib.s3gd_encode_vote2.argtypes = [vp, ctypes.c_int, u32, u64, u32p, vp]
    lib.s3gd_apply_vote2.restype = ctypes.c_int
    lib.s3gd_apply_vote2.argtypes = [vp, u32p, u64, ctypes.c_float, vp, vp]
    lib.s3gd_sparse_workspace_bytes.restype = sz
    lib.s3gd_sparse_workspace_bytes.argtypes = [u64]
    lib.s3gd_encode_vote_sparse.restype = ctypes.c_int
    lib.s3gd_encode_vote_sparse.argtypes = [vp, ctypes.c_int, u32, u64, u32, u32, u32p, vp, sz, vp]
    lib.s3gd_apply_vote_sparse.restype = ctypes.c_int
    lib.s3gd_apply_vote_sparse.argtypes = [vp, u32p, ctypes.c_int, u64, u32, u64, ctypes.c_float, vp, vp]
    f32, i32, i64, mat = ctypes.c_float, ctypes.c_int, ctypes.c_int64, ctypes.POINTER(Matrix)
    lib.s3gd_orthogonalise_workspace_bytes.restype = sz
    lib.s3gd_orthogonalise_workspace_bytes.argtypes = [i32, u64, u64]
    lib.s3gd_orthogonalise.restype = i32
    lib.s3gd_orthogonalise.argtypes = [mat, mat, i32, u64, u64, i32, f32, f32, f32, f32, i32, vp, sz, vp]
    lib.s3gd_step_ortho.restype = i32
    lib.s3gd_step_ortho.argtypes = [mat, mat, mat, i32, u64, u64, f32, i32, f32, f32, f32, i32, f32, f32, f32, f32, i32, vp, sz, vp]
    lib.s3gd_embed.restype = i32
    lib.s3gd_embed.argtypes = [vp, i32, i64, u64, u64, vp, i32, u64, f32, vp, i32, i64, vp, vp]
    lib.s3gd_embed_grad_workspace_bytes.restype = sz
    lib.s3gd_embed_grad_workspace_bytes.argtypes = [i32, u64, u64, u64]
    lib.s3gd_embed_grad.restype = i32
    lib.s3gd_embed_grad.argtypes = [vp, i32, i64, i64, vp, i32, i32, u64, u64, u64, f32, vp, i32, i64, i32, vp, vp, sz, vp]
    lib.s3gd_layer_norm.restype = i32
    lib.s3gd_layer_norm.argtypes = [vp, i32, i64, i64, vp, i64, i64, vp, i64, i64, vp, vp, i32, vp, i32, i32, u64, u64, f32, vp, i32, i64, i64, vp]
    lib.s3gd_layer_norm_grad_workspace_bytes.restype = sz
    lib.s3gd_layer_norm_grad_workspace_bytes.argtypes = [i32, u64, u64]
    lib.s3gd_layer_norm_grad.restype = i32
    lib.s3gd_layer_norm_grad.argtypes = [vp, i32, i64, i64, vp, i32, i64, i64, vp, i64, i64, vp, i32, vp, i32, i32, u64, u64, f32, vp, i64, i64,
                                         vp, vp, i32, i64, i32, vp, sz, vp]
    lib.s3gd_clip_workspace_bytes.restype = sz
    lib.s3gd_clip_workspace_bytes.argtypes = [i32]
    lib.s3gd_grad_norm.restype = i32
    lib.s3gd_grad_norm.argtypes = [vp, i32, i32, vp, vp, sz, vp]
    lib.s3gd_clip.restype = i32
    lib.s3gd_clip.argtypes = [vp, i32, i32, f32, f32, vp, vp, sz, vp]
    if path is None:
        _lib = lib
    return lib


def _ptr(t: Optional[torch.Tensor], dtype: torch.dtype, numel: Optional[int] = None, name: str = "tensor"):
    if t is None:
        return None
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.is_contiguous() and t.dtype == dtype):
        raise TypeError(f"{name} must be a contiguous CUDA tensor of dtype {dtype}")
    if numel is not None and t.numel() < numel:
        raise ValueError(f"{name} has {t.numel()} elements, needs {numel}")
    return ctypes.c_void_p(t.data_ptr())


def _stream(t: torch.Tensor):
    return ctypes.c_void_p(torch.cuda.current_stream(t.device).cuda_stream)


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream_of(index: int):
    """The current stream of a device as an address, without a Stream object in between (1 us less per call)."""
    return _raw_stream(index) if _raw_stream is not None else torch.cuda.current_stream(index).cuda_stream


_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


class _on:
    """torch.cuda.device of the tensors of a short call, which have to share one (None: not given); nothing is switched where it is
    current already."""

    __slots__ = ("index", "before")

    def __init__(self, t: torch.Tensor, *others: Optional[torch.Tensor]):
        self.index = index = t.get_device()
        for o in others:
            if o is not None and o.get_device() != index:
                raise TypeError(f"tensors of one call must be on one device, not on {t.device} and {o.device}")

    def __enter__(self):
        self.before = _current_device()
        if self.before != self.index:
            torch.cuda.set_device(self.index)

    def __exit__(self, *exc):
        if self.before != self.index:
            torch.cuda.set_device(self.before)


def _check(call: str, code: int) -> None:
    if code != S3GD_OK:
        raise S3gdError(call, code)


def s3gd_status_string(code: int) -> str:
    return load().s3gd_status_string(int(code)).decode()


def s3gd_workspace_bytes(M: int, d: int, K: int) -> int:
    return int(load().s3gd_workspace_bytes(int(M), int(d), int(K)))


def alloc_workspace(M: int, d: int, K: int, device="cuda") -> torch.Tensor:
    """A uint8 CUDA tensor of s3gd_workspace_bytes(M, d, K) bytes (torch allocations are 512-byte aligned)."""
    n = s3gd_workspace_bytes(M, d, K)
    if n == 0:
        raise ValueError("invalid (M, d, K)")
    return torch.empty(n, dtype=torch.uint8, device=device)


def words(K: int) -> int:
    return (int(K) + 31) // 32


def s3gd_topk_sign(grads: torch.Tensor, K: int, out_idx: torch.Tensor, out_signbits: torch.Tensor,
                   ws: torch.Tensor) -> None:
    """grads [M, d] fp32 -> out_idx [M, K] (uint32 values in int32 storage), out_signbits [M, ceil(K/32)]."""
    g = _ptr(grads, torch.float32, name="grads")
    M, d = grads.shape
    args = (g, M, d, K, _ptr(out_idx, torch.int32, M * K, "out_idx"),
            _ptr(out_signbits, torch.int32, M * words(K), "out_signbits"),
            _ptr(ws, torch.uint8, name="ws"), ws.numel())
    with _on(grads, out_idx, out_signbits, ws):
        code = load().s3gd_topk_sign(*args, _stream(grads))
    _check("s3gd_topk_sign", code)


def s3gd_majority_vote(idx: torch.Tensor, signbits: torch.Tensor, M: int, K: int, d: int,
                       out_vote: torch.Tensor, ws: torch.Tensor) -> None:
    """idx [M, K], signbits [M, ceil(K/32)] -> out_vote [d] int8 in {-1, 0, +1}."""
    args = (_ptr(idx, torch.int32, M * K, "idx"), _ptr(signbits, torch.int32, M * words(K), "signbits"), M, K, d,
            _ptr(out_vote, torch.int8, d, "out_vote"), _ptr(ws, torch.uint8, name="ws"), ws.numel())
    with _on(out_vote, idx, signbits, ws):
        code = load().s3gd_majority_vote(*args, _stream(out_vote))
    _check("s3gd_majority_vote", code)


def s3gd_apply(x: torch.Tensor, vote: torch.Tensor, lr: float) -> None:
    """x [d] fp32 updated in place by -lr * vote."""
    d = x.numel()
    args = (_ptr(x, torch.float32, name="x"), _ptr(vote, torch.int8, d, "vote"), d, ctypes.c_float(lr))
    with _on(x, vote):
        code = load().s3gd_apply(*args, _stream(x))
    _check("s3gd_apply", code)


def s3gd_step(x: torch.Tensor, grads: torch.Tensor, K: int, lr: float, ws: torch.Tensor,
              opt_idx: Optional[torch.Tensor] = None, opt_signbits: Optional[torch.Tensor] = None,
              opt_vote: Optional[torch.Tensor] = None) -> None:
    """The fused step: x [d] updated in place from grads [M, d]; optional outputs as in the unfused calls."""
    g = _ptr(grads, torch.float32, name="grads")
    M, d = grads.shape
    args = (_ptr(x, torch.float32, d, "x"), g, M, d, K, ctypes.c_float(lr),
            _ptr(opt_idx, torch.int32, M * K, "opt_idx"), _ptr(opt_signbits, torch.int32, M * words(K), "opt_signbits"),
            _ptr(opt_vote, torch.int8, d, "opt_vote"), _ptr(ws, torch.uint8, name="ws"), ws.numel())
    with _on(x, grads, opt_idx, opt_signbits, opt_vote, ws):
        code = load().s3gd_step(*args, _stream(x))
    _check("s3gd_step", code)


def s3gd_device_status(ws: torch.Tensor, raise_on_error: bool = True):
    """Synchronises the current stream; returns (status code, 8 diagnostic counters)."""
    info = (ctypes.c_uint32 * 8)()
    w = _ptr(ws, torch.uint8, name="ws")
    with torch.cuda.device(ws.device):
        code = load().s3gd_device_status(w, _stream(ws), info)
    if raise_on_error:
        _check("s3gd_device_status", code)
    return code, list(info)


def s3gd_last_device_status(ws: torch.Tensor) -> int:
    """Synchronises the current stream; returns the status code recorded by the kernels (0 = ok)."""
    w = _ptr(ws, torch.uint8, name="ws")
    with torch.cuda.device(ws.device):
        return int(load().s3gd_last_device_status(w, _stream(ws)))


def s3gd_debug_topk_sign(grads: torch.Tensor, K: int, out_idx: torch.Tensor, out_signbits: torch.Tensor,
                         ws: torch.Tensor, sample_rank: int) -> None:
    """s3gd_topk_sign with the sampling rank of the filter threshold forced (0: the library's own)."""
    g = _ptr(grads, torch.float32, name="grads")
    M, d = grads.shape
    args = (g, M, d, K, _ptr(out_idx, torch.int32, M * K, "out_idx"),
            _ptr(out_signbits, torch.int32, M * words(K), "out_signbits"),
            _ptr(ws, torch.uint8, name="ws"), ws.numel())
    with _on(grads, out_idx, out_signbits, ws):
        code = load().s3gd_debug_topk_sign(*args, _stream(grads), int(sample_rank))
    _check("s3gd_debug_topk_sign", code)


def s3gd_debug_step(x: torch.Tensor, grads: torch.Tensor, K: int, lr: float, ws: torch.Tensor, sample_rank: int,
                    opt_idx: Optional[torch.Tensor] = None, opt_signbits: Optional[torch.Tensor] = None,
                    opt_vote: Optional[torch.Tensor] = None, prevote_rank: int = 0) -> None:
    """s3gd_step with the sampling ranks of the two filter thresholds forced (0: the library's own)."""
    g = _ptr(grads, torch.float32, name="grads")
    M, d = grads.shape
    args = (_ptr(x, torch.float32, d, "x"), g, M, d, K, ctypes.c_float(lr),
            _ptr(opt_idx, torch.int32, M * K, "opt_idx"), _ptr(opt_signbits, torch.int32, M * words(K), "opt_signbits"),
            _ptr(opt_vote, torch.int8, d, "opt_vote"), _ptr(ws, torch.uint8, name="ws"), ws.numel())
    with _on(x, grads, opt_idx, opt_signbits, opt_vote, ws):
        code = load().s3gd_debug_step(*args, _stream(x), int(sample_rank), int(prevote_rank))
    _check("s3gd_debug_step", code)


def s3gd_vote_apply(x: torch.Tensor, msg: torch.Tensor, n_groups: int, group_stride: int, M_group: int, K: int,
                    lr: float, ws: torch.Tensor, opt_vote: Optional[torch.Tensor] = None) -> None:
    """Vote over a message gathered from n_groups senders (each piece: indices then sign words) fused with the update."""
    d = x.numel()
    need = (n_groups - 1) * group_stride + M_group * (K + words(K)) if n_groups > 0 else 0
    args = (_ptr(x, torch.float32, name="x"), _ptr(msg, torch.int32, need, "msg"), n_groups, group_stride, M_group, K, d,
            ctypes.c_float(lr), _ptr(opt_vote, torch.int8, d, "opt_vote"), _ptr(ws, torch.uint8, name="ws"), ws.numel())
    with _on(x, msg, opt_vote, ws):
        code = load().s3gd_vote_apply(*args, _stream(x))
    _check("s3gd_vote_apply", code)


def s3gd_vote_counts(idx: torch.Tensor, signbits: torch.Tensor, M: int, K: int, d: int, out_counts: torch.Tensor,
                     opt_bad_count: Optional[torch.Tensor] = None) -> None:
    """Vote sums of M workers into out_counts: uint8 [d_padded] (128 + sum) or int32 [d_padded] (sum)."""
    if out_counts.dtype == torch.uint8:
        per, p = 1, _ptr(out_counts, torch.uint8, d, "out_counts")
    else:
        per, p = 4, _ptr(out_counts, torch.int32, d, "out_counts")
    args = (_ptr(idx, torch.int32, M * K, "idx"), _ptr(signbits, torch.int32, M * words(K), "signbits"), M, K, d,
            out_counts.numel(), p, per, _ptr(opt_bad_count, torch.int32, 1, "opt_bad_count"))
    with _on(out_counts, idx, signbits, opt_bad_count):
        code = load().s3gd_vote_counts(*args, _stream(out_counts))
    _check("s3gd_vote_counts", code)


def s3gd_encode_vote2(src: torch.Tensor, out_words: torch.Tensor, n_summed: int = 1) -> None:
    """Two-bit form of the vote from int32 sums, from summed biased bytes (uint8) or from an int8 vote."""
    n = src.numel()
    if src.dtype == torch.int32:
        kind, p = 0, _ptr(src, torch.int32, name="src")
    elif src.dtype == torch.uint8:
        kind, p = 1, _ptr(src, torch.uint8, name="src")
    else:
        kind, p = 2, _ptr(src, torch.int8, name="src")
    args = (p, kind, n_summed, n, _ptr(out_words, torch.int32, (n + 15) // 16, "out_words"))
    with _on(src, out_words):
        code = load().s3gd_encode_vote2(*args, _stream(src))
    _check("s3gd_encode_vote2", code)


def s3gd_apply_vote2(x: torch.Tensor, words2: torch.Tensor, lr: float, opt_vote: Optional[torch.Tensor] = None) -> None:
    """x <- x - lr * vote with the vote in its two-bit form."""
    d = x.numel()
    args = (_ptr(x, torch.float32, name="x"), _ptr(words2, torch.int32, (d + 15) // 16, "words"), d, ctypes.c_float(lr),
            _ptr(opt_vote, torch.int8, d, "opt_vote"))
    with _on(x, words2, opt_vote):
        code = load().s3gd_apply_vote2(*args, _stream(x))
    _check("s3gd_apply_vote2", code)


def sparse_piece_words(cap: int) -> int:
    """uint32 words of one sparse message: its count, cap indices, ceil(cap / 32) sign words."""
    return 1 + int(cap) + words(cap)


def s3gd_sparse_workspace_bytes(n: int) -> int:
    return int(load().s3gd_sparse_workspace_bytes(int(n)))


def s3gd_encode_vote_sparse(src: torch.Tensor, out_piece: torch.Tensor, cap: int, ws: torch.Tensor,
                            index_base: int = 0, n_summed: int = 1) -> None:
    """Sparse form (count, ascending indices, sign words) of the votes in src: int32 sums, summed biased bytes or int8."""
    n = src.numel()
    if src.dtype == torch.int32:
        kind, p = 0, _ptr(src, torch.int32, name="src")
    elif src.dtype == torch.uint8:
        kind, p = 1, _ptr(src, torch.uint8, name="src")
    else:
        kind, p = 2, _ptr(src, torch.int8, name="src")
    args = (p, kind, n_summed, n, index_base, cap, _ptr(out_piece, torch.int32, sparse_piece_words(cap), "out_piece"),
            _ptr(ws, torch.uint8, name="ws"), ws.numel())
    with _on(src, out_piece, ws):
        code = load().s3gd_encode_vote_sparse(*args, _stream(src))
    _check("s3gd_encode_vote_sparse", code)


def s3gd_apply_vote_sparse(x: torch.Tensor, pieces: torch.Tensor, n_pieces: int, piece_stride: int, cap: int, lr: float,
                           opt_bad_count: Optional[torch.Tensor] = None) -> None:
    """x <- x - lr * vote from n_pieces sparse messages lying piece_stride words apart."""
    d = x.numel()
    need = (n_pieces - 1) * piece_stride + sparse_piece_words(cap)
    args = (_ptr(x, torch.float32, name="x"), _ptr(pieces, torch.int32, need, "pieces"), n_pieces, piece_stride, cap, d,
            ctypes.c_float(lr), _ptr(opt_bad_count, torch.int32, 1, "opt_bad_count"))
    with _on(x, pieces, opt_bad_count):
        code = load().s3gd_apply_vote_sparse(*args, _stream(x))
    _check("s3gd_apply_vote_sparse", code)


PHASES = ("sample", "filter", "threshold", "emit", "apply")


def s3gd_profile_begin(max_steps: int) -> None:
    _check("s3gd_profile_begin", load().s3gd_profile_begin(int(max_steps)))


def s3gd_profile_begin_filter(max_steps: int) -> None:
    """As s3gd_profile_begin, but only the filter pass is bracketed by events (the other phases read 0)."""
    _check("s3gd_profile_begin_filter", load().s3gd_profile_begin_filter(int(max_steps)))


def s3gd_profile_begin_filter_every(max_steps: int, every: int) -> None:
    """As s3gd_profile_begin_filter with only every `every`-th step recorded (at most max_steps of them)."""
    _check("s3gd_profile_begin_filter_every", load().s3gd_profile_begin_filter_every(int(max_steps), int(every)))


def s3gd_profile_end(max_steps: int):
    """Returns (per-step list of 5 phase durations in ms, kernels enqueued since s3gd_profile_begin)."""
    buf = (ctypes.c_float * (5 * max_steps))()
    n = ctypes.c_int(0)
    launches = ctypes.c_uint64(0)
    _check("s3gd_profile_end", load().s3gd_profile_end(buf, ctypes.byref(n), ctypes.byref(launches)))
    steps = [[buf[5 * i + k] for k in range(5)] for i in range(n.value)]
    return steps, int(launches.value)


def s3gd_noalloc_max_d() -> int:
    return int(load().s3gd_noalloc_max_d())


def s3gd_majority_vote_noalloc(idx: torch.Tensor, signbits: torch.Tensor, M: int, K: int, d: int,
                               out_vote: torch.Tensor, opt_bad_count: Optional[torch.Tensor] = None) -> None:
    """Majority vote whose counters live inside the library: no workspace argument, nothing allocated.

    For callers that cannot obtain device memory where they vote (see include/s3gd.h).  d must not
    exceed s3gd_noalloc_max_d(); calls on one device share the built-in counters, so do not overlap them.
    """
    args = (_ptr(idx, torch.int32, M * K, "idx"), _ptr(signbits, torch.int32, M * words(K), "signbits"), M, K, d,
            _ptr(out_vote, torch.int8, d, "out_vote"), _ptr(opt_bad_count, torch.int32, 1, "opt_bad_count"))
    with _on(out_vote, idx, signbits, opt_bad_count):
        code = load().s3gd_majority_vote_noalloc(*args, _stream(out_vote))
    _check("s3gd_majority_vote_noalloc", code)


def s3gd_step_ex(x: torch.Tensor, grads: torch.Tensor, K: int, lr: float, ws: torch.Tensor,
                 err: Optional[torch.Tensor] = None, eta: float = 1.0,
                 v: Optional[torch.Tensor] = None, mu: float = 0.0,
                 opt_idx: Optional[torch.Tensor] = None, opt_signbits: Optional[torch.Tensor] = None,
                 opt_vote: Optional[torch.Tensor] = None) -> None:
    """The fused step with optional error memory err [M, d] (updated in place) and momentum v [d]."""
    g = _ptr(grads, torch.float32, name="grads")
    M, d = grads.shape
    args = (_ptr(x, torch.float32, d, "x"), g, _ptr(err, torch.float32, M * d, "err"), ctypes.c_float(eta),
            _ptr(v, torch.float32, d, "v"), ctypes.c_float(mu), M, d, K, ctypes.c_float(lr),
            _ptr(opt_idx, torch.int32, M * K, "opt_idx"), _ptr(opt_signbits, torch.int32, M * words(K), "opt_signbits"),
            _ptr(opt_vote, torch.int8, d, "opt_vote"), _ptr(ws, torch.uint8, name="ws"), ws.numel())
    with _on(x, grads, err, v, opt_idx, opt_signbits, opt_vote, ws):
        code = load().s3gd_step_ex(*args, _stream(x))
    _check("s3gd_step_ex", code)


def s3gd_apply_momentum(x: torch.Tensor, v: torch.Tensor, vote: torch.Tensor, mu: float, lr: float) -> None:
    """v <- mu * v + vote; x <- x - lr * v, in place."""
    d = x.numel()
    args = (_ptr(x, torch.float32, name="x"), _ptr(v, torch.float32, d, "v"), _ptr(vote, torch.int8, d, "vote"), d,
            ctypes.c_float(mu), ctypes.c_float(lr))
    with _on(x, v, vote):
        code = load().s3gd_apply_momentum(*args, _stream(x))
    _check("s3gd_apply_momentum", code)


def s3gd_randk_sign(grads: torch.Tensor, K: int, seed: int, step: int, out_idx: torch.Tensor,
                    out_signbits: torch.Tensor, ws: torch.Tensor) -> None:
    """RandKSign: out_idx [M, K] = pi(0..K-1) per worker (generation order), out_signbits [M, ceil(K/32)]."""
    g = _ptr(grads, torch.float32, name="grads")
    M, d = grads.shape
    args = (g, M, d, K, seed & 0xFFFFFFFF, step & 0xFFFFFFFF, _ptr(out_idx, torch.int32, M * K, "out_idx"),
            _ptr(out_signbits, torch.int32, M * words(K), "out_signbits"),
            _ptr(ws, torch.uint8, name="ws"), ws.numel())
    with _on(grads, out_idx, out_signbits, ws):
        code = load().s3gd_randk_sign(*args, _stream(grads))
    _check("s3gd_randk_sign", code)


def s3gd_step_randk(x: torch.Tensor, grads: torch.Tensor, K: int, lr: float, seed: int, step: int, ws: torch.Tensor,
                    opt_idx: Optional[torch.Tensor] = None, opt_signbits: Optional[torch.Tensor] = None,
                    opt_vote: Optional[torch.Tensor] = None) -> None:
    """The fused step with RandKSign in place of TopKSign."""
    g = _ptr(grads, torch.float32, name="grads")
    M, d = grads.shape
    args = (_ptr(x, torch.float32, d, "x"), g, M, d, K, ctypes.c_float(lr), seed & 0xFFFFFFFF, step & 0xFFFFFFFF,
            _ptr(opt_idx, torch.int32, M * K, "opt_idx"), _ptr(opt_signbits, torch.int32, M * words(K), "opt_signbits"),
            _ptr(opt_vote, torch.int8, d, "opt_vote"), _ptr(ws, torch.uint8, name="ws"), ws.numel())
    with _on(x, grads, opt_idx, opt_signbits, opt_vote, ws):
        code = load().s3gd_step_randk(*args, _stream(x))
    _check("s3gd_step_randk", code)


_DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.int8: 2, torch.int32: 3, torch.int64: 4}
_REAL = (torch.float32, torch.bfloat16)
_REAL_CODES = {d: _DTYPES[d] for d in _REAL}
_INDEX_CODES = {d: _DTYPES[d] for d in (torch.int32, torch.int64)}
#: Coefficients of the quintic that five steps of are usually taken.
ORTHO_COEFFS = (3.4445, -4.7750, 2.0315)


def s3gd_orthogonalise_workspace_bytes(batch: int, rows: int, cols: int) -> int:
    return int(load().s3gd_orthogonalise_workspace_bytes(int(batch), int(rows), int(cols)))


def alloc_ortho_workspace(batch: int, rows: int, cols: int, device="cuda") -> torch.Tensor:
    """A uint8 CUDA tensor for s3gd_orthogonalise / s3gd_step_ortho on [batch, rows, cols] (batch 1: one matrix)."""
    n = s3gd_orthogonalise_workspace_bytes(batch, rows, cols)
    if n == 0:
        raise ValueError("invalid (batch, rows, cols)")
    return torch.empty(n, dtype=torch.uint8, device=device)


def _matrices(**tensors):
    """The named tensors ([rows, cols] or [batch, rows, cols], all of one shape) as s3gd_matrix, and (batch, rows, cols).

    Rows lie contiguous in all of them, or columns in all of them: the transposed problem is then passed on."""
    given = {k: t for k, t in tensors.items() if t is not None}
    first = next(iter(given.values()))
    for k, t in given.items():
        if not (isinstance(t, torch.Tensor) and t.is_cuda and t.device == first.device):
            raise TypeError(f"{k} must be a CUDA tensor on the device of the others")
        if t.dim() not in (2, 3) or t.shape != first.shape:
            raise ValueError(f"{k} has shape {tuple(t.shape)}, needs [rows, cols] or [batch, rows, cols] like the others")
    rows, cols = first.shape[-2:]

    def whole(t, inner, outer, n_inner, n_outer):       # unit stride inside, rows that do not run into each other
        return (t.stride(inner) == 1 or n_inner == 1) and (t.stride(outer) >= n_inner or n_outer == 1)

    if all(whole(t, -1, -2, cols, rows) for t in given.values()):
        outer = -2
    elif all(whole(t, -2, -1, rows, cols) for t in given.values()):
        outer, rows, cols = -1, cols, rows
    else:
        raise ValueError(" and ".join(given) + " must all have contiguous rows, or all contiguous columns")
    mats = {}
    for k, t in tensors.items():
        if t is None:
            mats[k] = None
            continue
        mats[k] = ctypes.byref(Matrix(t.data_ptr(), _DTYPES.get(t.dtype, -1), t.stride(outer) if rows > 1 else cols,
                                      t.stride(0) if t.dim() == 3 else 0))
    return mats, first.shape[0] if first.dim() == 3 else 1, rows, cols


def _of(t: Optional[torch.Tensor], dtypes, name: str) -> None:
    if t is not None and t.dtype not in dtypes:
        raise TypeError(f"{name} has dtype {t.dtype}, needs one of {', '.join(str(d) for d in dtypes)}")


def s3gd_orthogonalise(g: torch.Tensor, out: torch.Tensor, ws: torch.Tensor, steps: int = 5, coeffs=ORTHO_COEFFS,
                       eps: float = 1e-7, split_steps: int = -1) -> None:
    """out <- g with its singular values moved towards 1 by `steps` Newton-Schulz products, per matrix of the batch.

    g fp32, bf16 or an int8 vote; out fp32 or bf16, g itself allowed.  split_steps: of how many steps the products take
    operands of 22 bits instead of 11 (-1: all)."""
    m, batch, rows, cols = _matrices(g=g, out=out)
    _of(g, _REAL + (torch.int8,), "g")
    _of(out, _REAL, "out")
    a, b, c = coeffs
    w = _ptr(ws, torch.uint8, name="ws")
    with _on(out, ws):
        code = load().s3gd_orthogonalise(m["g"], m["out"], batch, rows, cols, steps, a, b, c, eps, split_steps, w, ws.numel(), _stream_of(out.device.index))
    _check("s3gd_orthogonalise", code)


def s3gd_step_ortho(x: torch.Tensor, g: torch.Tensor, lr: float, ws: torch.Tensor, v: Optional[torch.Tensor] = None,
                    mu: float = 0.95, nesterov: bool = True, weight_decay: float = 0.0, scale: float = 1.0, steps: int = 5,
                    coeffs=ORTHO_COEFFS, eps: float = 1e-7, split_steps: int = -1) -> None:
    """x <- (1 - lr weight_decay) x - lr scale orthogonalise(u), u from the momentum v <- mu v + g (v None: u = g); in place.

    x fp32 or bf16; v fp32; g fp32, bf16 or the int8 vote."""
    m, batch, rows, cols = _matrices(x=x, v=v, g=g)
    _of(x, _REAL, "x")
    _of(v, (torch.float32,), "v")
    _of(g, _REAL + (torch.int8,), "g")
    a, b, c = coeffs
    w = _ptr(ws, torch.uint8, name="ws")
    with _on(x, ws):
        code = load().s3gd_step_ortho(m["x"], m["v"], m["g"], batch, rows, cols, mu, int(nesterov), lr, weight_decay, scale, steps, a, b, c,
                                      eps, split_steps, w, ws.numel(), _stream_of(x.device.index))
    _check("s3gd_step_ortho", code)


def _rows(t: torch.Tensor, dtypes, name: str, dim: Optional[int] = None):
    """Checks a CUDA tensor whose last axis is contiguous."""
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dim() >= 1):
        raise TypeError(f"{name} must be a CUDA tensor")
    _of(t, dtypes, name)
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError(f"{name} must be contiguous along its last axis")
    if dim is not None and t.shape[-1] != dim:
        raise ValueError(f"{name} has rows of {t.shape[-1]}, needs {dim}")


def _ids(ids: torch.Tensor):
    if not (isinstance(ids, torch.Tensor) and ids.is_cuda and ids.is_contiguous() and ids.dtype in (torch.int32, torch.int64)):
        raise TypeError("ids must be a contiguous CUDA tensor of dtype int32 or int64")


def s3gd_embed(table: torch.Tensor, ids: torch.Tensor, out: torch.Tensor, scale: float = 1.0,
               opt_bad_count: Optional[torch.Tensor] = None) -> None:
    """out[..., :] <- scale * table[ids[...], :]; a negative id gives a zero row.  table [vocab, dim], out ids.shape + [dim]."""
    try:                                   # a call for one token takes 8 us, half of it here: look once, name the fault afterwards
        index = out.get_device()
        whole = index >= 0 and table.get_device() == index and ids.get_device() == index and ids.is_contiguous()
        codes = _REAL_CODES[table.dtype], _INDEX_CODES[ids.dtype], _REAL_CODES[out.dtype]
    except (AttributeError, KeyError):
        whole = False
    if not whole:
        _rows(table, _REAL, "table")
        _ids(ids)
        _rows(out, _REAL, "out")
        raise TypeError(f"table, ids and out must be on one device, not on {table.device}, {ids.device} and {out.device}")
    shape, n = out.shape, ids.numel()
    if table.dim() != 2 or len(shape) == 0 or shape[:-1] != ids.shape:
        raise ValueError(f"table must be [vocab, dim] and out {tuple(ids.shape)} + [dim]")
    vocab, dim = table.shape
    table_stride = out_stride = dim
    if not table.is_contiguous():
        _rows(table, _REAL, "table")
        table_stride = table.stride(0)
    if shape[-1] != dim or not out.is_contiguous():
        _rows(out, _REAL, "out", dim)
        if len(shape) != 2:
            raise ValueError("out must be contiguous, or [n, dim] with contiguous rows")
        out_stride = out.stride(0)
    bad = None if opt_bad_count is None else _ptr(opt_bad_count, torch.int32, 1, "opt_bad_count")
    if bad is not None and opt_bad_count.get_device() != index:
        raise TypeError(f"opt_bad_count must be on the device of out, {out.device}")
    args = (table.data_ptr(), codes[0], table_stride, vocab, dim, ids.data_ptr(), codes[1], n, scale, out.data_ptr(), codes[2], out_stride, bad)
    if _current_device() == index:
        code = load().s3gd_embed(*args, _stream_of(index))
    else:
        with _on(out):
            code = load().s3gd_embed(*args, _stream_of(index))
    if code:
        _check("s3gd_embed", code)


def s3gd_embed_grad_workspace_bytes(M: int, T: int, vocab: int, dim: int) -> int:
    return int(load().s3gd_embed_grad_workspace_bytes(int(M), int(T), int(vocab), int(dim)))


def alloc_embed_workspace(M: int, T: int, vocab: int, dim: int, device="cuda") -> torch.Tensor:
    """A uint8 CUDA tensor for s3gd_embed_grad of M workers with T tokens each."""
    n = s3gd_embed_grad_workspace_bytes(M, T, vocab, dim)
    if n == 0:
        raise ValueError("invalid (M, T, vocab, dim)")
    return torch.empty(n, dtype=torch.uint8, device=device)


def s3gd_embed_grad(dout: torch.Tensor, ids: torch.Tensor, grads: torch.Tensor, vocab: int, ws: torch.Tensor, scale: float = 1.0,
                    accumulate: bool = False, opt_bad_count: Optional[torch.Tensor] = None) -> None:
    """Each worker's gradient of the table: dout [M, T, dim], ids [M, T] -> the first vocab * dim entries of each row of grads.

    grads is [M, >= vocab * dim] (a column slice of the step's gradient buffer), [M, vocab, dim], or [vocab, dim] where dout is
    [T, dim] and ids [T] (one worker).  Negative ids are skipped; accumulate adds to what grads holds."""
    try:
        index = grads.get_device()
        whole = (index >= 0 and dout.get_device() == index and ids.get_device() == index and ids.is_contiguous() and dout.shape[:-1] == ids.shape
                 and ids.dim() in (1, 2))
        codes = _REAL_CODES[dout.dtype], _INDEX_CODES[ids.dtype], _REAL_CODES[grads.dtype]
    except (AttributeError, KeyError):
        whole = False
    if not whole:
        _rows(dout, _REAL, "dout")
        _ids(ids)
        _rows(grads, _REAL, "grads")
        if not dout.device == ids.device == grads.device:
            raise TypeError(f"dout, ids and grads must be on one device, not on {dout.device}, {ids.device} and {grads.device}")
        raise ValueError("dout must be [M, T, dim] with ids [M, T], or [T, dim] with ids [T]")
    several = ids.dim() == 2
    M, T, dim = (ids.shape[0] if several else 1), ids.shape[-1], dout.shape[-1]
    if dim > 1 and dout.stride(-1) != 1:
        raise ValueError("dout must be contiguous along its last axis")
    shape = grads.shape
    if len(shape) == ids.dim() + 1 and shape[-2:] == (vocab, dim):
        per, given, stride = vocab * dim, shape[0] if several else 1, grads.stride(0) if several else 0
        packed = grads.is_contiguous() or ((dim == 1 or grads.stride(-1) == 1) and (vocab == 1 or grads.stride(-2) == dim))
    elif len(shape) == 2:
        per, given, stride = shape[1], shape[0], grads.stride(0)
        packed = per == 1 or grads.stride(1) == 1
    else:
        per = given = stride = 0
        packed = False
    if not packed or given != M or per < vocab * dim:
        raise ValueError(f"grads must be [{M}, >= {vocab * dim}] or [{M}, {vocab}, {dim}], contiguous within a worker")
    bad = None if opt_bad_count is None else _ptr(opt_bad_count, torch.int32, 1, "opt_bad_count")
    w = _ptr(ws, torch.uint8, name="ws")
    if ws.get_device() != index or (bad is not None and opt_bad_count.get_device() != index):
        raise TypeError(f"ws and opt_bad_count must be on the device of grads, {grads.device}")
    args = (dout.data_ptr(), codes[0], dout.stride(-2), dout.stride(0) if several else 0, ids.data_ptr(), codes[1], M, T, vocab, dim, scale,
            grads.data_ptr(), codes[2], stride if M > 1 else vocab * dim, accumulate, bad, w, ws.numel())
    if _current_device() == index:
        code = load().s3gd_embed_grad(*args, _stream_of(index))
    else:
        with _on(grads):
            code = load().s3gd_embed_grad(*args, _stream_of(index))
    if code:
        _check("s3gd_embed_grad", code)


def _norm_shape(x: torch.Tensor):
    """(M, T, dim) of rows [T, dim] or [M, T, dim], or of any contiguous [..., dim]."""
    shape = x.shape
    if len(shape) == 2:
        return 1, shape[0], shape[1]
    if len(shape) == 3:
        return shape
    if len(shape) == 0:
        raise ValueError("x must be [..., dim]")
    return 1, x.numel() // shape[-1] if shape[-1] else 0, shape[-1]


def _norm_strides(t: Optional[torch.Tensor], like: torch.Tensor, name: str):
    """Elements from row to row and from worker to worker; (0, 0) where the tensor is not given."""
    if t is None:
        return 0, 0
    shape = t.shape
    if shape != like.shape:
        raise ValueError(f"{name} has shape {tuple(shape)}, needs {tuple(like.shape)}")
    if t.is_contiguous():
        return shape[-1], shape[-1] * shape[-2] if len(shape) > 2 else 0
    if len(shape) not in (2, 3):
        raise ValueError(f"{name} must be contiguous, or [T, dim] or [M, T, dim]")
    _rows(t, _REAL, name)
    return t.stride(-2), t.stride(0) if len(shape) == 3 else 0


def _norm_device(index: int, **tensors: Optional[torch.Tensor]):
    """Checks that the tensors given are CUDA tensors on one device, of types that the calls take."""
    for name, t in tensors.items():
        if t is None:
            continue
        if not (isinstance(t, torch.Tensor) and t.is_cuda):
            raise TypeError(f"{name} must be a CUDA tensor")
        if t.get_device() != index:
            raise TypeError(f"{name} must be on the device of the others, cuda:{index}, not on {t.device}")


def _norm_ids(ids: Optional[torch.Tensor], like: torch.Tensor):
    if ids is None:
        return None, 3
    _ids(ids)
    if ids.shape != like.shape[:-1]:
        raise ValueError(f"ids has shape {tuple(ids.shape)}, needs {tuple(like.shape[:-1])}")
    return ids.data_ptr(), _INDEX_CODES[ids.dtype]


def _param(t: Optional[torch.Tensor], dim: int, name: str):
    if t is None:
        return None
    if t.dim() != 1 or t.shape[0] != dim or (dim > 1 and t.stride(0) != 1):
        raise ValueError(f"{name} must be [{dim}], contiguous")
    return t.data_ptr()


def s3gd_layer_norm(x: torch.Tensor, y: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None,
                    eps: float = 1e-5, ids: Optional[torch.Tensor] = None, add: Optional[torch.Tensor] = None,
                    total: Optional[torch.Tensor] = None) -> None:
    """y[..., :] <- layer norm of x[..., :], or of total <- x + add where add and total are given.

    x, y (and add, total) are [T, dim] or [M, T, dim] with contiguous rows, or contiguous [..., dim]; fp32 or bf16, add and total
    of x's type.  ids (shape of x without its last axis): rows whose id is negative become zero."""
    args = _norm_args(x, y, weight, bias, eps, ids, add, total)
    index = x.get_device()
    if _current_device() == index:
        code = load().s3gd_layer_norm(*args, _stream_of(index))
    else:
        with _on(x):
            code = load().s3gd_layer_norm(*args, _stream_of(index))
    if code:
        _check("s3gd_layer_norm", code)


def _like(t: torch.Tensor, index: int, shape) -> bool:
    return t.get_device() == index and t.is_contiguous() and t.shape == shape


def _vector(t: Optional[torch.Tensor], index: int, dim: int):
    """The address of a contiguous [dim] on the device; None where it is not given; -1 where it is something else."""
    if t is None:
        return None
    return t.data_ptr() if t.get_device() == index and t.dim() == 1 and t.numel() == dim and t.is_contiguous() else -1


def _norm_args(x, y, weight, bias, eps, ids, add, total):
    """Arguments of s3gd_layer_norm.  A call for a few tokens is over in some microseconds: contiguous tensors are looked at once here,
    everything else, and what is wrong, below."""
    try:
        index, shape, kind = x.get_device(), x.shape, x.dtype
        dim = shape[-1]
        w, b = _vector(weight, index, dim), _vector(bias, index, dim)
        xd, yd = _REAL_CODES[kind], _REAL_CODES[y.dtype]
        pd = _REAL_CODES[weight.dtype if weight is not None else bias.dtype] if w or b else 0
        if (index >= 0 and dim > 0 and w != -1 and b != -1 and x.is_contiguous() and _like(y, index, shape)
                and (weight is None or bias is None or weight.dtype is bias.dtype)
                and ((add is None and total is None) or (add.dtype is kind and total.dtype is kind and _like(add, index, shape) and _like(total, index, shape)))
                and (ids is None or _like(ids, index, shape[:-1]))):
            i, it = (None, 3) if ids is None else (ids.data_ptr(), _INDEX_CODES[ids.dtype])
            p, q = (None, None) if add is None else (add.data_ptr(), total.data_ptr())
            return (x.data_ptr(), xd, dim, 0, p, dim, 0, q, dim, 0, w, b, pd, i, it, 1, x.numel() // dim, dim, eps, y.data_ptr(), yd, dim, 0)
    except (AttributeError, KeyError, IndexError):
        pass
    if not (isinstance(x, torch.Tensor) and x.is_cuda):
        raise TypeError("x must be a CUDA tensor")
    index = x.get_device()
    _norm_device(index, y=y, weight=weight, bias=bias, ids=ids, add=add, total=total)
    for t, name in ((x, "x"), (y, "y"), (weight, "weight"), (bias, "bias")):
        _of(t, _REAL, name)
    if y is None:
        raise TypeError("y must be a CUDA tensor")
    if weight is not None and bias is not None and weight.dtype != bias.dtype:
        raise TypeError(f"weight and bias must have one dtype, not {weight.dtype} and {bias.dtype}")
    if (add is None) != (total is None):
        raise ValueError("add and total come together")
    _of(add, (x.dtype,), "add")
    _of(total, (x.dtype,), "total")
    M, T, dim = _norm_shape(x)
    xs, xw = _norm_strides(x, x, "x")
    ys, yw = _norm_strides(y, x, "y")
    as_, aw = _norm_strides(add, x, "add")
    ts, tw = _norm_strides(total, x, "total")
    idp, idt = _norm_ids(ids, x)
    given = bias if weight is None else weight
    return (x.data_ptr(), _REAL_CODES[x.dtype], xs, xw, None if add is None else add.data_ptr(), as_, aw,
            None if total is None else total.data_ptr(), ts, tw, _param(weight, dim, "weight"), _param(bias, dim, "bias"),
            0 if given is None else _REAL_CODES[given.dtype], idp, idt, M, T, dim, eps, y.data_ptr(), _REAL_CODES[y.dtype], ys, yw)


def s3gd_layer_norm_grad_workspace_bytes(M: int, T: int, dim: int) -> int:
    return int(load().s3gd_layer_norm_grad_workspace_bytes(int(M), int(T), int(dim)))


def alloc_layer_norm_workspace(M: int, T: int, dim: int, device="cuda") -> torch.Tensor:
    """A uint8 CUDA tensor for s3gd_layer_norm_grad of M workers with T rows of dim each."""
    n = s3gd_layer_norm_grad_workspace_bytes(M, T, dim)
    if n == 0:
        raise ValueError("invalid (M, T, dim)")
    return torch.empty(n, dtype=torch.uint8, device=device)


def _worker_rows(t: Optional[torch.Tensor], M: int, dim: int, several: bool, name: str):
    """Elements from worker to worker of a gradient [M, dim] (or [dim] for one worker)."""
    if t is None:
        return None, 0
    shape = t.shape
    if shape == (M, dim):
        stride = t.stride(0)
    elif shape == (dim,) and not several:
        stride = dim
    else:
        raise ValueError(f"{name} has shape {tuple(shape)}, needs {(M, dim)}" + ("" if several else f" or {(dim,)}"))
    if dim > 1 and t.stride(-1) != 1:
        raise ValueError(f"{name} must be contiguous along its last axis")
    return t.data_ptr(), stride if M > 1 else dim


def s3gd_layer_norm_grad(dy: torch.Tensor, x: torch.Tensor, dx: Optional[torch.Tensor], weight: Optional[torch.Tensor],
                         dweight: Optional[torch.Tensor], dbias: Optional[torch.Tensor], ws: torch.Tensor, eps: float = 1e-5,
                         ids: Optional[torch.Tensor] = None, dtotal: Optional[torch.Tensor] = None, accumulate: bool = False) -> None:
    """Gradient of s3gd_layer_norm: dx (+ dtotal), and each worker's gradient of weight and bias.

    dy, x, dx, dtotal are [T, dim] or [M, T, dim]; x is what was normalised (total, where there was one); dx and dtotal have its
    type.  dweight and dbias are [M, dim] (columns of the workers' rows of a gradient buffer) or [dim] for one worker, of one
    type; accumulate adds to what they hold.  dx, or dweight and dbias, may be None; dx may be dy, x or dtotal itself."""
    args = _norm_grad_args(dy, x, dx, weight, dweight, dbias, ws, eps, ids, dtotal, accumulate)
    index = x.get_device()
    if _current_device() == index:
        code = load().s3gd_layer_norm_grad(*args, _stream_of(index))
    else:
        with _on(x):
            code = load().s3gd_layer_norm_grad(*args, _stream_of(index))
    if code:
        _check("s3gd_layer_norm_grad", code)


def _norm_grad_args(dy, x, dx, weight, dweight, dbias, ws, eps, ids, dtotal, accumulate):
    """Arguments of s3gd_layer_norm_grad, by the same two ways as _norm_args."""
    try:
        index, shape, kind = x.get_device(), x.shape, x.dtype
        M, T, dim = shape if len(shape) == 3 else (1, *shape)
        w, rows = _vector(weight, index, dim), (M, dim)
        stride = dweight.stride(0)
        if (index >= 0 and w != -1 and x.is_contiguous() and _like(dy, index, shape) and _like(dx, index, shape) and dx.dtype is kind
                and (dtotal is None or (_like(dtotal, index, shape) and dtotal.dtype is kind)) and (ids is None or _like(ids, index, shape[:-1]))
                and dweight.get_device() == index and dbias.get_device() == index and dweight.shape == rows and dbias.shape == rows
                and (dim == 1 or dweight.stride(1) == 1 == dbias.stride(1)) and dbias.stride(0) == stride and dweight.dtype is dbias.dtype
                and ws.get_device() == index and ws.dtype is torch.uint8 and ws.is_contiguous()):
            i, it = (None, 3) if ids is None else (ids.data_ptr(), _INDEX_CODES[ids.dtype])
            return (dy.data_ptr(), _REAL_CODES[dy.dtype], dim, T * dim, x.data_ptr(), _REAL_CODES[kind], dim, T * dim,
                    None if dtotal is None else dtotal.data_ptr(), dim, T * dim, w, 0 if w is None else _REAL_CODES[weight.dtype], i, it, M, T, dim,
                    eps, dx.data_ptr(), dim, T * dim, dweight.data_ptr(), dbias.data_ptr(), _REAL_CODES[dweight.dtype], stride if M > 1 else dim,
                    accumulate, ws.data_ptr(), ws.numel())
    except (AttributeError, KeyError, IndexError, ValueError):
        pass
    if not (isinstance(x, torch.Tensor) and x.is_cuda):
        raise TypeError("x must be a CUDA tensor")
    index = x.get_device()
    w = _ptr(ws, torch.uint8, name="ws")
    if dy is None or w is None:
        raise TypeError("dy and ws must be CUDA tensors")
    _norm_device(index, dy=dy, dx=dx, weight=weight, dweight=dweight, dbias=dbias, ws=ws, ids=ids, dtotal=dtotal)
    for t, name in ((dy, "dy"), (x, "x"), (weight, "weight"), (dweight, "dweight"), (dbias, "dbias")):
        _of(t, _REAL, name)
    if dweight is not None and dbias is not None and dweight.dtype != dbias.dtype:
        raise TypeError(f"dweight and dbias must have one dtype, not {dweight.dtype} and {dbias.dtype}")
    _of(dx, (x.dtype,), "dx")
    _of(dtotal, (x.dtype,), "dtotal")
    given = dbias if dweight is None else dweight
    if x.dim() not in (2, 3):
        raise ValueError("x must be [T, dim] or [M, T, dim]")
    if dx is None and (given is None or dtotal is not None):
        raise ValueError("dx must be given" + (" with dtotal" if dtotal is not None else ", or dweight or dbias"))
    M, T, dim = _norm_shape(x)
    xs, xw = _norm_strides(x, x, "x")
    ds, dw = _norm_strides(dy, x, "dy")
    os, ow = _norm_strides(dx, x, "dx")
    ts, tw = _norm_strides(dtotal, x, "dtotal")
    idp, idt = _norm_ids(ids, x)
    wp, stride = _worker_rows(dweight, M, dim, x.dim() == 3, "dweight")
    bp, bstride = _worker_rows(dbias, M, dim, x.dim() == 3, "dbias")
    if dweight is not None and dbias is not None and stride != bstride:
        raise ValueError(f"dweight and dbias must have one distance from worker to worker, not {stride} and {bstride}")
    return (dy.data_ptr(), _REAL_CODES[dy.dtype], ds, dw, x.data_ptr(), _REAL_CODES[x.dtype], xs, xw, None if dtotal is None else dtotal.data_ptr(), ts, tw,
            _param(weight, dim, "weight"), 0 if weight is None else _REAL_CODES[weight.dtype], idp, idt, M, T, dim, eps,
            None if dx is None else dx.data_ptr(), os, ow, wp, bp, 0 if given is None else _REAL_CODES[given.dtype], stride or bstride, accumulate, w, ws.numel())


def s3gd_clip_workspace_bytes(M: int) -> int:
    return int(load().s3gd_clip_workspace_bytes(int(M)))


def alloc_clip_workspace(M: int = 1, device="cuda") -> torch.Tensor:
    """A uint8 CUDA tensor for s3gd_grad_norm and s3gd_clip of M workers, whatever their tensors."""
    n = s3gd_clip_workspace_bytes(M)
    if n == 0:
        raise ValueError("invalid M")
    return torch.empty(n, dtype=torch.uint8, device=device)


def _in_one_piece(shape, strides) -> bool:
    """Whether the entries fill one piece of memory, in whatever order of axes."""
    expected = 1
    for stride, size in sorted(zip(strides, shape)):
        if size != 1:
            if stride != expected:
                return False
            expected *= size
    return True


_T = torch.Tensor
_dtype_of = operator.attrgetter("dtype")


def _once(places, entries, pointers=()) -> None:
    """Refuses an output that is named twice, or that lies in place of one gradient and is read as another one (pointers) too."""
    written = set(places)
    if len(written) != len(places):
        seen = [p for p, n in zip(places, entries) if n]
        if len(set(seen)) != len(seen):
            raise ValueError("an output is named twice: it would be scaled twice, or once, as it happens")
    if not written.isdisjoint(pointers):
        read = {p for p, o, n in zip(pointers, places, entries) if n and p != o}
        if any(n and o in read for o, n in zip(places, entries)):
            raise ValueError("an output is also read as another gradient: it would be read scaled or not, as it happens")


def _plain_parts(grads, outs, index: int, M: int, several: bool, writes: bool, apart: bool):
    """As _parts for lists of contiguous gradients of one type (and outputs of one type that lie alike); None for others.

    A list has hundreds of tensors and its kernels take some ten microseconds: each question is put to all tensors at once."""
    dtypes, devices = set(map(_dtype_of, grads)), set(map(_T.get_device, grads))
    sizes = list(map(_T.size, grads))
    if len(dtypes) != 1 or devices != {index} or not all(map(_T.is_contiguous, grads)) or (several and not all(s and s[0] == M for s in sizes)):
        return None
    code = _REAL_CODES[dtypes.pop()]
    entries, pointers = [n // M for n in map(_T.numel, grads)] if M > 1 else list(map(_T.numel, grads)), list(map(_T.data_ptr, grads))
    if outs is grads:
        if writes:
            _once(pointers, entries)
        return array.array("Q", chain.from_iterable(zip(pointers, pointers, entries, entries, entries, repeat(code | code << 32)))), len(pointers)
    dtypes = set(map(_dtype_of, outs))
    if len(dtypes) != 1 or set(map(_T.get_device, outs)) != devices or sizes != list(map(_T.size, outs)):
        return None
    distances = entries
    if not all(map(_T.is_contiguous, outs)):
        strides = list(map(_T.stride, outs))
        if not several or any(a[1:] != b[1:] for a, b in zip(strides, map(_T.stride, grads))):
            return None
        distances = [s[0] for s in strides]
    code |= _REAL_CODES[dtypes.pop()] << 32
    places = list(map(_T.data_ptr, outs))
    _once(places, entries, pointers if apart else ())
    return array.array("Q", chain.from_iterable(zip(pointers, places, entries, entries, distances, repeat(code)))), len(pointers)


def _parts(grads, out, index: int, M: int, several: bool, writes: bool, apart: bool = False):
    """The tensors as an array of s3gd_part, and their number; apart: an output may be in place, but not read as another gradient."""
    if isinstance(grads, torch.Tensor):
        grads, out = (grads,), (out,) if isinstance(out, torch.Tensor) else out
    grads = list(grads)
    outs = grads if out is None else list(out)
    if len(outs) != len(grads):
        raise ValueError(f"{len(outs)} outputs for {len(grads)} gradients")
    plain = None
    if len(grads) > 3:                                   # (a tensor by itself takes 3.6 us below and 5.9 above)
        try:
            plain = _plain_parts(grads, outs, index, M, several, writes, apart)
        except (TypeError, AttributeError, KeyError):    # something that is no tensor, or of another type: named below
            pass
    if plain is not None:
        return plain
    packed, first = array.array("Q"), 1 if several else 0
    for i, (g, o) in enumerate(zip(grads, outs)):
        try:
            if g.get_device() != index or o.get_device() != index:
                raise TypeError(f"tensors of one call must be on one device: gradient {i} or its output is not on cuda:{index}")
            code = _REAL_CODES[g.dtype] | _REAL_CODES[o.dtype] << 32
        except (AttributeError, KeyError):
            for t in (g, o):
                if not (isinstance(t, torch.Tensor) and t.is_cuda):
                    raise TypeError(f"gradient {i} and its output must be CUDA tensors") from None
                _of(t, _REAL, f"gradient {i} or its output")
        shape = g.shape
        if several and (len(shape) == 0 or shape[0] != M):
            raise ValueError(f"gradient {i} has shape {tuple(shape)}, needs {M} workers in front")
        n = g.numel() // M
        if n == 0:
            continue
        strides = g.stride()
        if not g.is_contiguous() and not _in_one_piece(shape[first:], strides[first:]):
            raise ValueError(f"gradient {i} is not in one piece" + (" within a worker" if several else ""))
        out_strides = strides
        if o is not g:
            out_strides = o.stride()
            if o.shape != shape:
                raise ValueError(f"output {i} has shape {tuple(o.shape)}, needs {tuple(shape)}")
            if out_strides[first:] != strides[first:] and any(a != b and s != 1 for a, b, s in zip(out_strides[first:], strides[first:], shape[first:])):
                raise ValueError(f"output {i} does not lie like its gradient: strides {out_strides} and {strides}")
        packed.extend((g.data_ptr(), o.data_ptr(), n, strides[0] if several else 0, out_strides[0] if several else 0, code))
    if writes:
        _once(packed[1::6].tolist(), packed[2::6], packed[::6] if apart else ())
    return packed, len(packed) // 6


def _norms(norm: torch.Tensor):
    if not (isinstance(norm, torch.Tensor) and norm.is_cuda and norm.dtype == torch.float32 and norm.dim() <= 1 and norm.is_contiguous()):
        raise TypeError("norm must be a contiguous CUDA tensor of dtype float32, [] or [M]")
    several = norm.dim() == 1
    if norm.numel() == 0:
        raise ValueError("norm must have an entry for each of at least one worker")
    return norm.get_device(), norm.numel(), several


def _clip_room(ws: torch.Tensor, index: int):
    if not (isinstance(ws, torch.Tensor) and ws.is_cuda and ws.dtype == torch.uint8 and ws.is_contiguous()):
        raise TypeError("ws must be a contiguous CUDA tensor of dtype torch.uint8")
    if ws.get_device() != index:
        raise TypeError(f"ws must be on the device of norm, cuda:{index}, not on {ws.device}")
    return ws.data_ptr(), ws.numel()


def s3gd_grad_norm(grads, norm: torch.Tensor, ws: torch.Tensor) -> None:
    """norm <- the norm over all entries of the tensors in grads (one tensor, or a sequence).

    norm is fp32: [] for one norm over everything, or [M] for one per worker, where every tensor's first axis is the M workers.
    Tensors are fp32 or bf16, each in one piece (within a worker)."""
    index, M, several = _norms(norm)
    packed, count = _parts(grads, None, index, M, several, False)
    args = (packed.buffer_info()[0] if count else None, count, M, norm.data_ptr(), *_clip_room(ws, index))
    if _current_device() == index:
        code = load().s3gd_grad_norm(*args, _stream_of(index))
    else:
        with _on(norm):
            code = load().s3gd_grad_norm(*args, _stream_of(index))
    if code:
        _check("s3gd_grad_norm", code)


def s3gd_clip(grads, max_norm: float, norm: torch.Tensor, ws: torch.Tensor, out=None, eps: float = 1e-6) -> None:
    """out <- grads * min(1, max_norm / (norm + eps)), norm as s3gd_grad_norm gives it; per worker where norm is [M].

    out (None: in place) has a tensor for each of grads, of the same shape and order of axes, fp32 or bf16: e.g. the columns of a
    gradient buffer, out[i] = rows[:, a:b].unflatten(1, shape).  Outputs overlap no other tensor of the call, and none is named twice
    (refused where they begin at one place)."""
    index, M, several = _norms(norm)
    packed, count = _parts(grads, out, index, M, several, True, True)
    args = (packed.buffer_info()[0] if count else None, count, M, max_norm, eps, norm.data_ptr(), *_clip_room(ws, index))
    if _current_device() == index:
        code = load().s3gd_clip(*args, _stream_of(index))
    else:
        with _on(norm):
            code = load().s3gd_clip(*args, _stream_of(index))
    if code:
        _check("s3gd_clip", code)
