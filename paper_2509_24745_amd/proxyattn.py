"""Python binding of libproxyattn.so (argument marshalling only).

The functions here carry the C ABI's names and arguments (see
include/proxyattn.h).  Tensors are torch tensors on the GPU; only their
device pointers and the current HIP stream cross the boundary.  Every step
of the path runs in the library's HIP kernels: there is no fallback, and the
module raises ImportError when the library has not been built.
"""
from __future__ import annotations

import ctypes
import math
import os
from dataclasses import dataclass, replace
from functools import cached_property

import torch  # loaded first: the library then binds to torch's HIP runtime

_HERE = os.path.dirname(os.path.abspath(__file__))
# PROXYATTN_LIBRARY selects another build of the library (the sanitized host
# build for the boundary tests); by default the one next to this file
LIB_PATH = os.environ.get("PROXYATTN_LIBRARY") or os.path.join(_HERE, "libproxyattn.so")

BF16 = 0
F32 = 1

E_OK, E_INVALID, E_UNSUPPORTED, E_WORKSPACE, E_HIP = 0, 1, 2, 3, 4
TOPK_CONSTANT, TOPK_ROW_RATIO, LIST_ASCENDING = 0, 1, 2
LIST_BAD_COUNT, LIST_BAD_INDEX, LIST_DUPLICATE = 1, 2, 4
CACHE_SAME, CACHE_FP4 = 0, 1


class proxyattn_problem(ctypes.Structure):
    _fields_ = [
        ("struct_size", ctypes.c_uint32),
        ("seq_len", ctypes.c_int32),
        ("num_q_heads", ctypes.c_int32),
        ("num_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("block_size", ctypes.c_int32),
        ("num_proxy_groups", ctypes.c_int32),
        ("stride", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
        ("softmax_scale", ctypes.c_float),
        ("q_tok_stride", ctypes.c_int64),
        ("q_head_stride", ctypes.c_int64),
        ("kv_tok_stride", ctypes.c_int64),
        ("kv_head_stride", ctypes.c_int64),
        ("o_tok_stride", ctypes.c_int64),
        ("o_head_stride", ctypes.c_int64),
        ("attn_order", ctypes.c_int32),
        ("attn_chunk_rows", ctypes.c_int32),
    ]


class proxyattn_rotary(ctypes.Structure):
    _fields_ = [
        ("struct_size", ctypes.c_uint32),
        ("rotary_dim", ctypes.c_int32),
        ("interleaved", ctypes.c_int32),
        ("table_len", ctypes.c_int32),
        ("norm_eps", ctypes.c_double),
        ("cos", ctypes.c_void_p),
        ("sin", ctypes.c_void_p),
        ("q_weight", ctypes.c_void_p),
        ("k_weight", ctypes.c_void_p),
        ("q_out_tok_stride", ctypes.c_int64),
        ("q_out_head_stride", ctypes.c_int64),
        ("k_out_tok_stride", ctypes.c_int64),
        ("k_out_head_stride", ctypes.c_int64),
    ]


class proxyattn_cache(ctypes.Structure):
    _fields_ = [
        ("struct_size", ctypes.c_uint32),
        ("num_seqs", ctypes.c_int32),
        ("num_tokens", ctypes.c_int32),
        ("max_new", ctypes.c_int32),
        ("max_len", ctypes.c_int32),
        ("num_q_heads", ctypes.c_int32),
        ("num_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("page_size", ctypes.c_int32),
        ("num_pages", ctypes.c_int32),
        ("table_width", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
        ("cache_type", ctypes.c_int32),
        ("softmax_scale", ctypes.c_float),
        ("q_tok_stride", ctypes.c_int64),
        ("q_head_stride", ctypes.c_int64),
        ("kv_tok_stride", ctypes.c_int64),
        ("kv_head_stride", ctypes.c_int64),
        ("o_tok_stride", ctypes.c_int64),
        ("o_head_stride", ctypes.c_int64),
    ]


_SIGS = {
    "proxyattn_workspace_size": [ctypes.c_void_p, ctypes.c_void_p],
    "proxyattn_workspace_layout": [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p],
    "proxyattn_estimate": [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                           ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p],
    "proxyattn_select_budget": [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_float,
                                ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                ctypes.c_void_p],
    "proxyattn_budget": [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_float, ctypes.c_int32,
                         ctypes.c_void_p, ctypes.c_void_p],
    "proxyattn_select_topk": [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int32,
                              ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p],
    "proxyattn_head_overlap": [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int32,
                               ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_void_p,
                               ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p],
    "proxyattn_check_lists": [ctypes.c_void_p] * 5,
    "proxyattn_block_sparse_prefill": [ctypes.c_void_p] * 9 + [ctypes.c_size_t, ctypes.c_void_p],
    "proxyattn_dense_prefill": [ctypes.c_void_p] * 7 + [ctypes.c_size_t, ctypes.c_void_p],
    "proxyattn_kv_blocked_size": [ctypes.c_void_p, ctypes.c_void_p],
    "proxyattn_prepare_kv": [ctypes.c_void_p] * 4 + [ctypes.c_size_t, ctypes.c_void_p],
    "proxyattn_blocked_workspace_size": [ctypes.c_void_p, ctypes.c_void_p],
    "proxyattn_block_sparse_prefill_blocked": [ctypes.c_void_p] * 3 + [ctypes.c_size_t]
                                              + [ctypes.c_void_p] * 5
                                              + [ctypes.c_size_t, ctypes.c_void_p],
    "proxyattn_dense_prefill_blocked": [ctypes.c_void_p] * 3 + [ctypes.c_size_t]
                                       + [ctypes.c_void_p] * 3 + [ctypes.c_size_t, ctypes.c_void_p],
    "proxyattn_block_sparse_prefill_blocked_noalloc": [ctypes.c_void_p] * 3 + [ctypes.c_size_t]
                                                      + [ctypes.c_void_p] * 5,
    "proxyattn_norm_rotate": [ctypes.c_void_p] * 5 + [ctypes.c_int32] + [ctypes.c_void_p] * 3,
    "proxyattn_cache_size": [ctypes.c_void_p] * 3,
    "proxyattn_cache_append": [ctypes.c_void_p] * 14,
    "proxyattn_cache_read": [ctypes.c_void_p] * 11,
    "proxyattn_cache_workspace_size": [ctypes.c_void_p] * 2,
    "proxyattn_cache_attention": [ctypes.c_void_p] * 12 + [ctypes.c_size_t, ctypes.c_void_p],
    "proxyattn_error_string": [ctypes.c_int],
    "proxyattn_last_error": [],
    "proxyattn_version": [],
}
EXPORTS = tuple(_SIGS)


def load_library(path: str = LIB_PATH) -> ctypes.CDLL:
    if not os.path.exists(path):
        raise ImportError(f"{path} is missing: build it with `python -m paper_2509_24745_amd.build`")
    lib = ctypes.CDLL(path)
    for name, args in _SIGS.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = ctypes.c_char_p if name in ("proxyattn_error_string", "proxyattn_last_error",
                                                 "proxyattn_version") else ctypes.c_int
    return lib


_lib = None


def lib() -> ctypes.CDLL:
    global _lib
    if _lib is None:
        _lib = load_library()
    return _lib


class ProxyAttnError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"{msg} (code {code})")
        self.code = code


def _check(rc: int):
    if rc != E_OK:
        L = lib()
        raise ProxyAttnError(rc, f"{L.proxyattn_error_string(rc).decode()}: "
                                 f"{L.proxyattn_last_error().decode()}")


@dataclass(frozen=True)
class Problem:
    """Host-side problem description (mirrors proxyattn_problem)."""

    seq_len: int
    num_q_heads: int
    num_kv_heads: int
    head_dim: int
    block_size: int
    num_proxy_groups: int
    stride: int = 4
    dtype: str = "bf16"
    softmax_scale: float = 0.0
    q_tok_stride: int = 0
    q_head_stride: int = 0
    kv_tok_stride: int = 0
    kv_head_stride: int = 0
    o_tok_stride: int = 0
    o_head_stride: int = 0
    attn_order: int = 0        # 0 by kernel and size; 1 plain, 2 row chunks, 3 KV-head-major chunks then short rows
    attn_chunk_rows: int = 0   # 0 by size

    @property
    def num_blocks(self) -> int:
        return -(-self.seq_len // self.block_size)

    @property
    def scale(self) -> float:
        return self.softmax_scale if self.softmax_scale > 0 else 1.0 / math.sqrt(self.head_dim)

    @property
    def torch_dtype(self):
        return torch.bfloat16 if self.dtype == "bf16" else torch.float32

    @cached_property
    def _rotated(self):
        """What proxyattn_norm_rotate looks at: rows of q and of k, the struct."""
        n, hq, hkv, d = self.seq_len, self.num_q_heads, self.num_kv_heads, self.head_dim
        return (_Rows(n, hq, d, self.q_tok_stride, self.q_head_stride),
                _Rows(n, hkv, d, self.kv_tok_stride, self.kv_head_stride),
                ctypes.byref(self.c_struct()))

    def c_struct(self) -> proxyattn_problem:
        p = proxyattn_problem()
        p.struct_size = ctypes.sizeof(proxyattn_problem)
        p.seq_len = self.seq_len
        p.num_q_heads = self.num_q_heads
        p.num_kv_heads = self.num_kv_heads
        p.head_dim = self.head_dim
        p.block_size = self.block_size
        p.num_proxy_groups = self.num_proxy_groups
        p.stride = self.stride
        p.dtype = BF16 if self.dtype == "bf16" else (F32 if self.dtype == "fp32" else 99)
        p.softmax_scale = self.softmax_scale
        p.q_tok_stride, p.q_head_stride = self.q_tok_stride, self.q_head_stride
        p.kv_tok_stride, p.kv_head_stride = self.kv_tok_stride, self.kv_head_stride
        p.o_tok_stride, p.o_head_stride = self.o_tok_stride, self.o_head_stride
        p.attn_order, p.attn_chunk_rows = self.attn_order, self.attn_chunk_rows
        return p


def _ptr(x) -> int | None:
    if x is None:
        return None
    if isinstance(x, int):
        return x
    return x.data_ptr()


def _nbytes(x) -> int:
    return x.numel() * x.element_size()


def _stream(stream) -> int | None:
    if stream is None:
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def proxyattn_workspace_size(prob: Problem) -> int:
    n = ctypes.c_size_t(0)
    p = prob.c_struct()
    _check(lib().proxyattn_workspace_size(ctypes.byref(p), ctypes.byref(n)))
    return n.value


def proxyattn_kv_blocked_size(prob: Problem) -> int:
    n = ctypes.c_size_t(0)
    p = prob.c_struct()
    _check(lib().proxyattn_kv_blocked_size(ctypes.byref(p), ctypes.byref(n)))
    return n.value


def proxyattn_blocked_workspace_size(prob: Problem) -> int:
    n = ctypes.c_size_t(0)
    p = prob.c_struct()
    _check(lib().proxyattn_blocked_workspace_size(ctypes.byref(p), ctypes.byref(n)))
    return n.value


def proxyattn_workspace_layout(prob: Problem):
    a, b = ctypes.c_size_t(0), ctypes.c_size_t(0)
    p = prob.c_struct()
    _check(lib().proxyattn_workspace_layout(ctypes.byref(p), ctypes.byref(a), ctypes.byref(b)))
    return a.value, b.value


# Checks of torch arguments: the library receives raw pointers and cannot see
# the allocations, so a tensor smaller than the problem would be read or
# written out of bounds, and a host tensor's address would reach a kernel as
# if it were device memory.  Each check needs the number of elements the call
# touches from the tensor's data pointer (ints are raw pointers and are passed
# through unchecked).  Q, K, V and O may be strided views (the problem carries
# their strides); every other array is read as packed, so it must be
# contiguous.
def _need(x, n_elems: int, name: str, dtype=None, contiguous: bool = True):
    if x is None or isinstance(x, int) or n_elems <= 0:
        return
    if dtype is not None and x.dtype != dtype:
        raise ProxyAttnError(E_INVALID, f"{name}: dtype {x.dtype}, the problem needs {dtype}")
    avail = x.untyped_storage().nbytes() // x.element_size() - x.storage_offset()
    if avail < n_elems:
        raise ProxyAttnError(E_INVALID, f"{name}: {avail} elements from its data pointer, the "
                                        f"problem touches {n_elems}")
    if contiguous and not x.is_contiguous():
        raise ProxyAttnError(E_INVALID, f"{name}: not contiguous (read as a packed array)")
    if not x.is_cuda:
        raise ProxyAttnError(E_INVALID, f"{name}: tensor on {x.device}, the library needs "
                                        f"device memory of the current GPU")
    if x.device.index != torch.cuda.current_device():
        raise ProxyAttnError(E_INVALID, f"{name}: tensor on {x.device}, the current device is "
                                        f"cuda:{torch.cuda.current_device()}")


def _need_ws(workspace, n_bytes: int, name: str = "workspace"):
    """A workspace of at least n_bytes on the current GPU (sizes are checked
    again by the library against what the problem needs)."""
    if workspace is None or isinstance(workspace, int):
        return
    _need(workspace, 1, name)
    if workspace.numel() * workspace.element_size() < n_bytes:
        raise ProxyAttnError(E_WORKSPACE, f"{name}: {workspace.numel() * workspace.element_size()}"
                                          f" bytes, the problem needs {n_bytes}")


def _span(n, heads, d, tok_stride, head_stride):
    tok = tok_stride or heads * d
    head = head_stride or d
    return (n - 1) * tok + (heads - 1) * head + d if n > 0 else 0


def _need_q(prob: Problem, q, name="q"):
    _need(q, _span(prob.seq_len, prob.num_q_heads, prob.head_dim, prob.q_tok_stride,
                   prob.q_head_stride), name, prob.torch_dtype, contiguous=False)


def _need_kv(prob: Problem, x, name):
    _need(x, _span(prob.seq_len, prob.num_kv_heads, prob.head_dim, prob.kv_tok_stride,
                   prob.kv_head_stride), name, prob.torch_dtype, contiguous=False)


def _need_out(prob: Problem, out):
    _need(out, _span(prob.seq_len, prob.num_q_heads, prob.head_dim, prob.o_tok_stride,
                     prob.o_head_stride), "out", prob.torch_dtype, contiguous=False)


def _need_scores(prob: Problem, block_logscore):
    mq = prob.num_blocks
    _need(block_logscore, prob.num_proxy_groups * mq * mq, "block_logscore", torch.float32)


def _need_lists(prob: Problem, block_count, block_index):
    mq = prob.num_blocks
    _need(block_count, prob.num_q_heads * mq, "block_count", torch.int32)
    _need(block_index, prob.num_q_heads * mq * mq, "block_index", torch.int32)


def proxyattn_estimate(prob: Problem, q, k, block_logscore, lastblk_mass, workspace, stream=None):
    _need_q(prob, q)
    _need_kv(prob, k, "k")
    _need_scores(prob, block_logscore)
    _need(lastblk_mass, prob.num_q_heads * prob.num_blocks, "lastblk_mass", torch.float32)
    _need_ws(workspace, 0)
    p = prob.c_struct()
    _check(lib().proxyattn_estimate(ctypes.byref(p), _ptr(q), _ptr(k), _ptr(block_logscore),
                                    _ptr(lastblk_mass), _ptr(workspace), _nbytes(workspace)
                                    if workspace is not None else 0, _stream(stream)))


def proxyattn_select_budget(prob: Problem, block_logscore, lastblk_mass, gamma: float,
                            min_budget_tokens: int, head_count, block_count, block_index,
                            stream=None):
    _need_scores(prob, block_logscore)
    _need(lastblk_mass, prob.num_q_heads * prob.num_blocks, "lastblk_mass", torch.float32)
    _need(head_count, prob.num_q_heads, "head_count", torch.int32)
    _need_lists(prob, block_count, block_index)
    p = prob.c_struct()
    _check(lib().proxyattn_select_budget(ctypes.byref(p), _ptr(block_logscore), _ptr(lastblk_mass),
                                         float(gamma), int(min_budget_tokens), _ptr(head_count),
                                         _ptr(block_count), _ptr(block_index), _stream(stream)))


def proxyattn_budget(prob: Problem, lastblk_mass, gamma: float, min_budget_tokens: int, head_count,
                     stream=None):
    _need(lastblk_mass, prob.num_q_heads * prob.num_blocks, "lastblk_mass", torch.float32)
    _need(head_count, prob.num_q_heads, "head_count", torch.int32)
    p = prob.c_struct()
    _check(lib().proxyattn_budget(ctypes.byref(p), _ptr(lastblk_mass), float(gamma),
                                  int(min_budget_tokens), _ptr(head_count), _stream(stream)))


def proxyattn_select_topk(prob: Problem, block_logscore, head_count, mode: int, block_count,
                          block_index, stream=None):
    _need_scores(prob, block_logscore)
    _need(head_count, prob.num_q_heads, "head_count", torch.int32)
    _need_lists(prob, block_count, block_index)
    p = prob.c_struct()
    _check(lib().proxyattn_select_topk(ctypes.byref(p), _ptr(block_logscore), _ptr(head_count),
                                       int(mode), _ptr(block_count), _ptr(block_index),
                                       _stream(stream)))


def proxyattn_head_overlap(prob: Problem, q, k, query_token: int, topk: int, sink_tokens: int,
                           renormalize: bool, scores, workspace, stream=None):
    _need_q(prob, q)
    _need_kv(prob, k, "k")
    _need(scores, prob.num_q_heads * prob.num_q_heads, "scores", torch.float32)
    _need_ws(workspace, 0)
    p = prob.c_struct()
    _check(lib().proxyattn_head_overlap(ctypes.byref(p), _ptr(q), _ptr(k), int(query_token),
                                        int(topk), int(sink_tokens), int(bool(renormalize)),
                                        _ptr(scores), _ptr(workspace),
                                        _nbytes(workspace) if workspace is not None else 0,
                                        _stream(stream)))


def proxyattn_check_lists(prob: Problem, block_count, block_index, status, stream=None):
    _need_lists(prob, block_count, block_index)
    _need(status, prob.num_q_heads * prob.num_blocks, "status", torch.int32)
    p = prob.c_struct()
    _check(lib().proxyattn_check_lists(ctypes.byref(p), _ptr(block_count), _ptr(block_index),
                                       _ptr(status), _stream(stream)))


def proxyattn_block_sparse_prefill(prob: Problem, q, k, v, block_count, block_index, out, lse,
                                   workspace, stream=None):
    _need_q(prob, q)
    _need_kv(prob, k, "k")
    _need_kv(prob, v, "v")
    _need_lists(prob, block_count, block_index)
    _need_out(prob, out)
    _need(lse, prob.num_q_heads * prob.seq_len, "lse", torch.float32)
    _need_ws(workspace, 0)
    p = prob.c_struct()
    _check(lib().proxyattn_block_sparse_prefill(
        ctypes.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(block_count), _ptr(block_index),
        _ptr(out), _ptr(lse), _ptr(workspace),
        _nbytes(workspace) if workspace is not None else 0, _stream(stream)))


def proxyattn_dense_prefill(prob: Problem, q, k, v, out, lse, workspace, stream=None):
    _need_q(prob, q)
    _need_kv(prob, k, "k")
    _need_kv(prob, v, "v")
    _need_out(prob, out)
    _need(lse, prob.num_q_heads * prob.seq_len, "lse", torch.float32)
    _need_ws(workspace, 0)
    p = prob.c_struct()
    _check(lib().proxyattn_dense_prefill(
        ctypes.byref(p), _ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse), _ptr(workspace),
        _nbytes(workspace) if workspace is not None else 0, _stream(stream)))


def _need_kvb(prob: Problem, kv_blocked):
    if kv_blocked is None or isinstance(kv_blocked, int):
        return
    _need_ws(kv_blocked, proxyattn_kv_blocked_size(prob), "kv_blocked")


def proxyattn_prepare_kv(prob: Problem, k, v, kv_blocked, stream=None):
    _need_kv(prob, k, "k")
    _need_kv(prob, v, "v")
    _need_kvb(prob, kv_blocked)
    p = prob.c_struct()
    _check(lib().proxyattn_prepare_kv(ctypes.byref(p), _ptr(k), _ptr(v), _ptr(kv_blocked),
                                      _nbytes(kv_blocked) if kv_blocked is not None else 0,
                                      _stream(stream)))


def proxyattn_block_sparse_prefill_blocked(prob: Problem, q, kv_blocked, block_count, block_index,
                                           out, lse, workspace, stream=None):
    _need_q(prob, q)
    _need_kvb(prob, kv_blocked)
    _need_lists(prob, block_count, block_index)
    _need_out(prob, out)
    _need(lse, prob.num_q_heads * prob.seq_len, "lse", torch.float32)
    _need_ws(workspace, 0)
    p = prob.c_struct()
    _check(lib().proxyattn_block_sparse_prefill_blocked(
        ctypes.byref(p), _ptr(q), _ptr(kv_blocked),
        _nbytes(kv_blocked) if kv_blocked is not None else 0, _ptr(block_count),
        _ptr(block_index), _ptr(out), _ptr(lse), _ptr(workspace),
        _nbytes(workspace) if workspace is not None else 0, _stream(stream)))


def proxyattn_block_sparse_prefill_blocked_noalloc(prob: Problem, q, kv_blocked, block_count,
                                                   block_index, out, lse, stream=None):
    _need_q(prob, q)
    _need_kvb(prob, kv_blocked)
    _need_lists(prob, block_count, block_index)
    _need_out(prob, out)
    _need(lse, prob.num_q_heads * prob.seq_len, "lse", torch.float32)
    p = prob.c_struct()
    _check(lib().proxyattn_block_sparse_prefill_blocked_noalloc(
        ctypes.byref(p), _ptr(q), _ptr(kv_blocked),
        _nbytes(kv_blocked) if kv_blocked is not None else 0, _ptr(block_count),
        _ptr(block_index), _ptr(out), _ptr(lse), _stream(stream)))


def proxyattn_dense_prefill_blocked(prob: Problem, q, kv_blocked, out, lse, workspace,
                                    stream=None):
    _need_q(prob, q)
    _need_kvb(prob, kv_blocked)
    _need_out(prob, out)
    _need(lse, prob.num_q_heads * prob.seq_len, "lse", torch.float32)
    _need_ws(workspace, 0)
    p = prob.c_struct()
    _check(lib().proxyattn_dense_prefill_blocked(
        ctypes.byref(p), _ptr(q), _ptr(kv_blocked),
        _nbytes(kv_blocked) if kv_blocked is not None else 0, _ptr(out), _ptr(lse),
        _ptr(workspace), _nbytes(workspace) if workspace is not None else 0, _stream(stream)))


# ---------------------------------------------------------------------------
# around the prefill: norm and rotation, and the paged cache
# ---------------------------------------------------------------------------
# A decode step is a few launches of some microseconds, so these calls check
# their tensors with as few queries as will do and keep their C structs.
def _arg(x, n_elems: int, name: str, dtype, device: int, contiguous: bool = True) -> int | None:
    """Checks a torch argument as _need does and returns its pointer (ints and
    None as they are)."""
    if x is None or type(x) is int:
        return x
    if not (x.dtype is dtype and x.is_contiguous() and x.numel() >= n_elems
            and x.get_device() == device >= 0):
        _need(x, n_elems, name, dtype, contiguous)   # says what is wrong, or that nothing is
    return x.data_ptr()


class _Rows:
    """Token rows [n][heads][d] with strides (0: packed) as a call reads or writes them."""

    __slots__ = ("shape", "stride", "span")

    def __init__(self, n, heads, d, tok_stride, head_stride):
        self.shape = (n, heads, d)
        self.stride = (tok_stride or heads * d, head_stride or d, 1)
        self.span = _span(n, heads, d, tok_stride, head_stride)

    def arg(self, x, name: str, dtype, device: int) -> int | None:
        """As _arg; a tensor of just this shape and these strides is looked at once."""
        if x is None or type(x) is int:
            return x
        if not (x.dtype is dtype and x.shape == self.shape and x.stride() == self.stride
                and x.get_device() == device >= 0):
            _need(x, self.span, name, dtype, contiguous=False)
        return x.data_ptr()


_gpu_seen = False


def _device_and_stream(stream) -> tuple[int, int | None]:
    """The current device (-1: none) and the stream's handle."""
    global _gpu_seen
    if not _gpu_seen:
        _gpu_seen = torch.cuda.is_available()
        if not _gpu_seen:
            return -1, stream if stream is None or isinstance(stream, int) else stream.cuda_stream
    dev = torch.cuda.current_device()
    if stream is None:   # torch.cuda.current_stream() makes a Stream first, which takes longer
        return dev, torch._C._cuda_getCurrentRawStream(dev)
    return dev, stream if isinstance(stream, int) else stream.cuda_stream


def _same(tensors, checked) -> bool:
    """Whether tensors that a descriptor holds still lie where they were checked."""
    return checked is not None and checked == tuple(_ptr(x) for x in tensors)


@dataclass(frozen=True, eq=False)
class Rotary:
    """Norm of each head and rotation by position (mirrors proxyattn_rotary).

    cos, sin: fp32 [table_len, rotary_dim / 2] on the GPU (with rotary_dim);
    q_weight, k_weight: [head_dim] in the problem's dtype, None for no norm."""

    rotary_dim: int = 0
    interleaved: bool = False
    eps: float = 1e-6
    cos: torch.Tensor | None = None
    sin: torch.Tensor | None = None
    q_weight: torch.Tensor | None = None
    k_weight: torch.Tensor | None = None
    q_out_tok_stride: int = 0
    q_out_head_stride: int = 0
    k_out_tok_stride: int = 0
    k_out_head_stride: int = 0

    @property
    def table_len(self) -> int:
        return self.cos.shape[0] if self.cos is not None else 0

    @property
    def _c(self):
        r = proxyattn_rotary()
        r.struct_size = ctypes.sizeof(proxyattn_rotary)
        r.rotary_dim, r.interleaved = self.rotary_dim, int(self.interleaved)
        r.table_len, r.norm_eps = self.table_len, self.eps
        r.cos, r.sin = _ptr(self.cos), _ptr(self.sin)
        r.q_weight, r.k_weight = _ptr(self.q_weight), _ptr(self.k_weight)
        r.q_out_tok_stride, r.q_out_head_stride = self.q_out_tok_stride, self.q_out_head_stride
        r.k_out_tok_stride, r.k_out_head_stride = self.k_out_tok_stride, self.k_out_head_stride
        return r

    def _out_rows(self, n: int, hq: int, hkv: int, d: int) -> tuple[_Rows, _Rows]:
        """Rows of the outputs."""
        held = self.__dict__.get("_rows")
        if held is None or held[0] != (n, hq, hkv, d):
            held = ((n, hq, hkv, d),
                    (_Rows(n, hq, d, self.q_out_tok_stride, self.q_out_head_stride),
                     _Rows(n, hkv, d, self.k_out_tok_stride, self.k_out_head_stride)))
            self.__dict__["_rows"] = held
        return held[1]

    def _arg(self, d: int, dtype, device: int):
        """The struct, by reference; its tensors checked once for a use (and
        again should they have moved)."""
        key, tensors = (d, dtype, device), (self.cos, self.sin, self.q_weight, self.k_weight)
        held = self.__dict__.get("_held")
        if held is not None and held[0] == key and _same(tensors, held[1]):
            return held[2]
        if self.rotary_dim > 0:
            if (self.cos is not None and self.sin is not None
                    and self.cos.shape[0] != self.sin.shape[0]):
                raise ProxyAttnError(E_INVALID, f"sin: {self.sin.shape[0]} rows, cos has "
                                                f"{self.table_len}")
            n = self.table_len * (self.rotary_dim // 2)
            _arg(self.cos, n, "cos", torch.float32, device)
            _arg(self.sin, n, "sin", torch.float32, device)
        _arg(self.q_weight, d, "q_weight", dtype, device)
        _arg(self.k_weight, d, "k_weight", dtype, device)
        ref = ctypes.byref(self._c)
        self.__dict__["_held"] = (key, tuple(_ptr(x) for x in tensors), ref)
        return ref


def proxyattn_norm_rotate(prob: Problem, rotary: Rotary, q, k, positions, first_position: int,
                          q_out, k_out, stream=None):
    dev, st = _device_and_stream(stream)
    n, hq, hkv, d = prob.seq_len, prob.num_q_heads, prob.num_kv_heads, prob.head_dim
    dt = prob.torch_dtype
    qr, kr, p = prob._rotated
    r = qo = ko = None
    if rotary is not None:
        r = rotary._arg(d, dt, dev)
        qor, kor = rotary._out_rows(n, hq, hkv, d)
        qo, ko = qor.arg(q_out, "q_out", dt, dev), kor.arg(k_out, "k_out", dt, dev)
    _check(lib().proxyattn_norm_rotate(p, r, qr.arg(q, "q", dt, dev), kr.arg(k, "k", dt, dev),
                                       _arg(positions, n, "positions", torch.int32, dev),
                                       int(first_position), qo, ko, st))


@dataclass(frozen=True)
class Cache:
    """A paged cache and a call's batch (mirrors proxyattn_cache)."""

    num_seqs: int
    num_tokens: int
    max_new: int
    max_len: int
    num_q_heads: int
    num_kv_heads: int
    head_dim: int
    page_size: int
    num_pages: int
    table_width: int
    dtype: str = "bf16"
    cache_type: str = "same"   # "same" (the dtype) or "fp4"
    softmax_scale: float = 0.0
    q_tok_stride: int = 0
    q_head_stride: int = 0
    kv_tok_stride: int = 0
    kv_head_stride: int = 0
    o_tok_stride: int = 0
    o_head_stride: int = 0

    @cached_property
    def torch_dtype(self):
        return torch.bfloat16 if self.dtype == "bf16" else torch.float32

    @cached_property
    def page_dtype(self):
        return torch.uint8 if self.cache_type == "fp4" else self.torch_dtype

    @cached_property
    def _ref(self):
        return ctypes.byref(self._c)

    @cached_property
    def _c(self):
        c = proxyattn_cache()
        c.struct_size = ctypes.sizeof(proxyattn_cache)
        for name in ("num_seqs", "num_tokens", "max_new", "max_len", "num_q_heads",
                     "num_kv_heads", "head_dim", "page_size", "num_pages", "table_width",
                     "softmax_scale", "q_tok_stride", "q_head_stride", "kv_tok_stride",
                     "kv_head_stride", "o_tok_stride", "o_head_stride"):
            setattr(c, name, getattr(self, name))
        c.dtype = {"bf16": BF16, "fp32": F32}.get(self.dtype, 99)
        c.cache_type = {"same": CACHE_SAME, "fp4": CACHE_FP4}.get(self.cache_type, 99)
        return c

    @cached_property
    def _sizes(self):
        """Rows of q, of k and v and of out; elements of a page pool and of its scales."""
        t, hq, hkv, d = self.num_tokens, self.num_q_heads, self.num_kv_heads, self.head_dim
        rows = self.num_pages * hkv * self.page_size
        fp4 = self.cache_type == "fp4"
        return (_Rows(t, hq, d, self.q_tok_stride, self.q_head_stride),
                _Rows(t, hkv, d, self.kv_tok_stride, self.kv_head_stride),
                _Rows(t, hq, d, self.o_tok_stride, self.o_head_stride),
                rows * (d // 2 if fp4 else d), rows * (d // 32) if fp4 else 0)

    @cached_property
    def _packed_q(self) -> "Cache":
        """The same with packed queries and outputs (a decode step's own)."""
        strides = dict(q_tok_stride=0, q_head_stride=0, o_tok_stride=0, o_head_stride=0)
        return replace(self, **strides)

    @cached_property
    def _workspace_bytes(self) -> int:
        return proxyattn_cache_workspace_size(self)


def proxyattn_cache_size(cache: Cache) -> tuple[int, int]:
    """Bytes of k_pages (and of v_pages) and of k_scales (and of v_scales)."""
    a, b = ctypes.c_size_t(0), ctypes.c_size_t(0)
    _check(lib().proxyattn_cache_size(cache._ref, ctypes.byref(a), ctypes.byref(b)))
    return a.value, b.value


def proxyattn_cache_workspace_size(cache: Cache) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().proxyattn_cache_workspace_size(cache._ref, ctypes.byref(n)))
    return n.value


@dataclass(frozen=True, eq=False)
class Pages:
    """The pools of a cache: k, v [num_pages, Hkv, page_size, d] (fp4: uint8
    [..., d / 2]) and, with fp4, k_scales, v_scales uint8 [num_pages, Hkv, d / 32,
    page_size]."""

    k: torch.Tensor
    v: torch.Tensor
    k_scales: torch.Tensor | None = None
    v_scales: torch.Tensor | None = None

    @classmethod
    def empty(cls, cache: Cache, device="cuda") -> "Pages":
        lead = (cache.num_pages, cache.num_kv_heads)
        fp4 = cache.cache_type == "fp4"
        row = cache.head_dim // 2 if fp4 else cache.head_dim
        pools = [torch.empty((*lead, cache.page_size, row), dtype=cache.page_dtype, device=device)
                 for _ in range(2)]
        if fp4:
            pools += [torch.empty((*lead, cache.head_dim // 32, cache.page_size),
                                  dtype=torch.uint8, device=device) for _ in range(2)]
        return cls(*pools)

    def _args(self, cache: Cache, device: int):
        """Pointers of the pools, checked once for a size (and again should
        they have moved)."""
        _, _, _, pool, scales = cache._sizes
        key = (pool, scales, cache.page_dtype, device)
        tensors = (self.k, self.v, self.k_scales, self.v_scales)
        held = self.__dict__.get("_held")
        if held is not None and held[0] == key and _same(tensors, held[1]):
            return held[1]
        ptrs = (_arg(self.k, pool, "k_pages", cache.page_dtype, device),
                _arg(self.v, pool, "v_pages", cache.page_dtype, device),
                _arg(self.k_scales, scales, "k_scales", torch.uint8, device),
                _arg(self.v_scales, scales, "v_scales", torch.uint8, device))
        self.__dict__["_held"] = (key, ptrs)
        return ptrs


def _arg_batch(cache: Cache, page_table, seq_lens, new_start, pages: Pages, device: int):
    """Pointers of page_table, seq_lens, new_start and the four pools."""
    b, i32 = cache.num_seqs, torch.int32
    return (_arg(page_table, b * cache.table_width, "page_table", i32, device),
            _arg(seq_lens, b, "seq_lens", i32, device),
            _arg(new_start, b + 1, "new_start", i32, device), *pages._args(cache, device))


def proxyattn_cache_append(cache: Cache, rotary: Rotary | None, q, k, v, q_out, page_table,
                           seq_lens, new_start, pages: Pages, stream=None):
    dev, st = _device_and_stream(stream)
    dt = cache.torch_dtype
    qr, kvr, _, _, _ = cache._sizes
    r = None
    if rotary is not None:
        r = rotary._arg(cache.head_dim, dt, dev)
        rows = rotary._out_rows(cache.num_tokens, cache.num_q_heads, cache.num_kv_heads,
                                cache.head_dim)[0]
        qo = rows.arg(q_out, "q_out", dt, dev)
    else:
        qo = _ptr(q_out)   # refused by the library
    args = (qr.arg(q, "q", dt, dev), kvr.arg(k, "k", dt, dev), kvr.arg(v, "v", dt, dev), qo)
    batch = _arg_batch(cache, page_table, seq_lens, new_start, pages, dev)
    _check(lib().proxyattn_cache_append(cache._ref, r, *args, *batch, st))


def proxyattn_cache_read(cache: Cache, page_table, seq_lens, new_start, pages: Pages, k_out,
                         v_out, stream=None):
    dev, st = _device_and_stream(stream)
    dt, kvr = cache.torch_dtype, cache._sizes[1]
    outs = (kvr.arg(k_out, "k_out", dt, dev), kvr.arg(v_out, "v_out", dt, dev))
    batch = _arg_batch(cache, page_table, seq_lens, new_start, pages, dev)
    _check(lib().proxyattn_cache_read(cache._ref, *batch, *outs, st))


def proxyattn_cache_attention(cache: Cache, q, page_table, seq_lens, new_start, pages: Pages, out,
                              lse, workspace, stream=None):
    dev, st = _device_and_stream(stream)
    dt = cache.torch_dtype
    qr, _, outr, _, _ = cache._sizes
    qp = qr.arg(q, "q", dt, dev)
    batch = _arg_batch(cache, page_table, seq_lens, new_start, pages, dev)
    op = outr.arg(out, "out", dt, dev)
    lp = _arg(lse, cache.num_q_heads * cache.num_tokens, "lse", torch.float32, dev)
    need = ws_bytes = cache._workspace_bytes
    if isinstance(workspace, torch.Tensor):
        ws_bytes = _nbytes(workspace)
        if not (ws_bytes >= need and workspace.get_device() == dev >= 0 and workspace.is_contiguous()):
            _need_ws(workspace, need)
        workspace = workspace.data_ptr()
    elif workspace is None:
        ws_bytes = 0
    _check(lib().proxyattn_cache_attention(cache._ref, qp, *batch, op, lp, workspace, ws_bytes,
                                           st))


def proxyattn_version() -> str:
    return lib().proxyattn_version().decode()


class Buffers:
    """Device buffers for one problem (allocation through torch only)."""

    def __init__(self, prob: Problem, device="cuda"):
        g, mq, hq = prob.num_proxy_groups, prob.num_blocks, prob.num_q_heads
        n, d = prob.seq_len, prob.head_dim
        f32, i32 = torch.float32, torch.int32
        self.prob = prob
        self.workspace = torch.empty(max(proxyattn_workspace_size(prob), 16), dtype=torch.uint8,
                                     device=device)
        self.logscore = torch.empty((g, mq, mq), dtype=f32, device=device)
        self.mass = torch.empty((hq, mq), dtype=f32, device=device)
        self.head_count = torch.empty(hq, dtype=i32, device=device)
        self.block_count = torch.empty((hq, mq), dtype=i32, device=device)
        self.block_index = torch.empty((hq, mq, mq), dtype=i32, device=device)
        self.out = torch.empty((n, hq, d), dtype=prob.torch_dtype, device=device)
        self.lse = torch.empty((hq, n), dtype=f32, device=device)


def prefill(prob: Problem, q, k, v, gamma: float, min_budget_tokens: int = 0,
            bufs: Buffers | None = None, stream=None, rotary: Rotary | None = None) -> Buffers:
    """Run the three steps (estimate, select_budget, block_sparse_prefill).  With a
    rotary, q and k are projections of tokens 0, 1, ..: they are normed and rotated
    in place first (its output strides have to be the problem's), and stay so should a
    later step refuse its arguments."""
    bufs = bufs or Buffers(prob, q.device)
    if rotary is not None:
        proxyattn_norm_rotate(prob, rotary, q, k, None, 0, q, k, stream)
    proxyattn_estimate(prob, q, k, bufs.logscore, bufs.mass, bufs.workspace, stream)
    proxyattn_select_budget(prob, bufs.logscore, bufs.mass, gamma, min_budget_tokens,
                            bufs.head_count, bufs.block_count, bufs.block_index, stream)
    proxyattn_block_sparse_prefill(prob, q, k, v, bufs.block_count, bufs.block_index, bufs.out,
                                   bufs.lse, bufs.workspace, stream)
    return bufs


class CacheBuffers:
    """What a decode step of one cache writes besides its pages."""

    def __init__(self, cache: Cache, device="cuda"):
        t, hq, d = cache.num_tokens, cache.num_q_heads, cache.head_dim
        self.cache = cache
        self.workspace = torch.empty(max(cache._workspace_bytes, 16), dtype=torch.uint8,
                                     device=device)
        self.q = torch.empty((t, hq, d), dtype=cache.torch_dtype, device=device)
        self.out = torch.empty((t, hq, d), dtype=cache.torch_dtype, device=device)
        self.lse = torch.empty((hq, t), dtype=torch.float32, device=device)


def decode(cache: Cache, rotary: Rotary, q, k, v, page_table, seq_lens, new_start, pages: Pages,
           bufs: CacheBuffers | None = None, stream=None) -> CacheBuffers:
    """One layer's step after the prefill: the batch's new tokens normed,
    rotated and appended, then their attention over the cache (cache_append,
    cache_attention).  The rotary's q_out strides and the cache's o strides are
    the packed ones."""
    bufs = bufs or CacheBuffers(cache, q.device)
    proxyattn_cache_append(cache, rotary, q, k, v, bufs.q, page_table, seq_lens, new_start, pages,
                           stream)
    packed = cache._packed_q
    proxyattn_cache_attention(packed, bufs.q, page_table, seq_lens, new_start, pages, bufs.out,
                              bufs.lse, bufs.workspace, stream)
    return bufs
