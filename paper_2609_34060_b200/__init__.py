"""Python binding of the KV-correction CUDA library (``libkvc.so``).

Argument marshalling only: torch tensors supply device memory and the stream,
every step of the path runs in the library's kernels.  The functions carry the
C ABI's names (``include/kvc.h``) and raise :class:`KvcError` on a non-zero
status.  There is no CPU fallback: if the shared object is missing or cannot
be loaded, the first call raises.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
from typing import List, Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libkvc.so")

KVC_CONTIG, KVC_PAGED = 0, 1
KVC_F32, KVC_BF16 = 0, 1
KVC_ROPE_HALF, KVC_ROPE_INTERLEAVED = 0, 1
KVC_PROJECT, KVC_FIT, KVC_FIT_FAST = 0, 1, 2
(KVC_SOLVER_SUBSPACE, KVC_SOLVER_FULL_RANK, KVC_SOLVER_FULL_DEPENDENT, KVC_SOLVER_FULL_SLOW, KVC_SOLVER_FULL_NO_GAP,
 KVC_SOLVER_FULL_SWEEPS) = (0, -1, 2, 3, 4, 5)
KVC_PATH_AUTO, KVC_PATH_GENERIC, KVC_PATH_TC, KVC_PATH_MIXED = 0, 1, 2, 3
KVC_MAX_SEGMENTS, KVC_COORDS_TARGET, KVC_COORDS_SOURCE = 16, 0, 1
KVC_GROUP_HEAD, KVC_GROUP_LAYER = 0, 1
KVC_FLAG_BAD_PAGE, KVC_FLAG_WAIT_EXPIRED, KVC_FLAG_NOT_CONVERGED, KVC_FLAG_BAD_LENGTH = 1, 2, 4, 8
KVC_FLAG_BAD_TREE, KVC_FLAG_BAD_PROB = 16, 32
KVC_TREE_MAX_Q = 1024
KVC_OK = 0
(KVC_E_INVALID_ARG, KVC_E_SHAPE, KVC_E_UNSUPPORTED, KVC_E_ALIAS, KVC_E_CUDA, KVC_E_WORKSPACE, KVC_E_DEVICE_FLAG,
 KVC_E_TOO_LARGE) = (-1, -2, -3, -4, -5, -6, -7, -8)

EXPORTS = (
    "kvc_apply", "kvc_chain", "kvc_state_update", "kvc_state_update_noalloc", "kvc_workspace_bytes", "kvc_apply_batch",
    "kvc_batch_workspace_bytes", "kvc_status_poll", "kvc_status_reset", "kvc_set_path", "kvc_last_path",
    "kvc_apply_bytes", "kvc_update_bytes", "kvc_strerror", "kvc_version", "kvc_gate_distance", "kvc_gate_weights",
    "kvc_apply_multi", "kvc_multi_workspace_bytes", "kvc_token_weights", "kvc_token_weights_workspace_bytes",
    "kvc_state_realign", "kvc_effective_rank", "kvc_fit_eigenvalues", "kvc_fit_solver", "kvc_group_fit_eigenvalues", "kvc_group_fit_solver", "kvc_selftest_wait_expiry", "kvc_apply_segmented", "kvc_state_update_segmented", "kvc_state_update_check", "kvc_state_update_chain",
    "kvc_chain_update_workspace_bytes", "kvc_chain_update_edge_stride", "kvc_chain_fused", "kvc_chain_workspace_bytes",
    "kvc_quantize", "kvc_dequantize", "kvc_append", "kvc_append_q8", "kvc_attend", "kvc_attend_q8", "kvc_attend_workspace_bytes",
    "kvc_tree_build", "kvc_append_rotated", "kvc_append_rotated_q8", "kvc_attend_tree", "kvc_attend_tree_q8", "kvc_verify", "kvc_keep", "kvc_keep_q8",
)


class KvcError(RuntimeError):
    def __init__(self, code: int, what: str):
        super().__init__(f"{what}: {strerror(code)} ({code})")
        self.code = code


class kvc_cache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("layout", C.c_int32), ("L", C.c_int32), ("H", C.c_int32),
                ("T", C.c_int32), ("d", C.c_int32), ("page_size", C.c_int32), ("n_phys_pages", C.c_int32),
                ("page_table", C.c_void_p), ("s_layer", C.c_int64), ("s_page", C.c_int64), ("s_head", C.c_int64),
                ("s_tok", C.c_int64)]


class kvc_state(C.Structure):
    _fields_ = [("coeff_k", C.c_void_p), ("coeff_v", C.c_void_p), ("basis_k", C.c_void_p), ("basis_v", C.c_void_p),
                ("r", C.c_int32), ("n_cov", C.c_int32), ("basis_dtype", C.c_int32), ("grouping", C.c_int32)]


class kvc_rope(C.Structure):
    _fields_ = [("theta", C.c_double), ("pairing", C.c_int32), ("reserved", C.c_int32), ("inv_freq", C.c_void_p)]


class kvc_segments(C.Structure):
    _fields_ = [("n", C.c_int32), ("t_begin", C.POINTER(C.c_int32)), ("shift", C.POINTER(C.c_int32)), ("coords", C.c_int32)]


class kvc_item(C.Structure):
    _fields_ = [("src", kvc_cache), ("dst", kvc_cache), ("st", kvc_state), ("shift", C.c_int32),
                ("t_begin", C.c_int32), ("t_end", C.c_int32), ("reserved", C.c_int32)]


class kvc_qcache(C.Structure):
    _fields_ = [("codes", kvc_cache), ("scale_k", C.c_void_p), ("scale_v", C.c_void_p), ("e_layer", C.c_int64),
                ("e_page", C.c_int64), ("e_head", C.c_int64), ("e_tok", C.c_int64)]


class kvc_requests(C.Structure):
    _fields_ = [("n", C.c_int32), ("max_q", C.c_int32), ("max_kv", C.c_int32), ("table_stride", C.c_int32),
                ("q_begin", C.c_void_p), ("kv_len", C.c_void_p), ("page_table", C.c_void_p)]


class kvc_heads(C.Structure):
    _fields_ = [("data", C.c_void_p), ("n_rows", C.c_int32), ("n_heads", C.c_int32), ("s_row", C.c_int64), ("s_head", C.c_int64)]


class kvc_tree(C.Structure):
    _fields_ = [("words", C.c_int32), ("n_rows", C.c_int32), ("parent", C.c_void_p), ("mask", C.c_void_p), ("depth", C.c_void_p)]


class kvc_rotary(C.Structure):
    _fields_ = [("rope", kvc_rope), ("amplitude", C.c_double), ("rot_dim", C.c_int32), ("reserved", C.c_int32), ("depth", C.c_void_p),
                ("pos_begin", C.c_void_p)]


class kvc_probs(C.Structure):
    _fields_ = [("p", C.c_void_p), ("n_rows", C.c_int32), ("n", C.c_int32), ("s_row", C.c_int64)]


_lib = None


def load(path: Optional[str] = None):
    """Load the shared library (once).  Raises if it is not there: no fallback."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or LIB_PATH
    if not os.path.exists(p):
        raise RuntimeError(f"{p} not found: build it with `python -m paper_2609_34060_b200.build`")
    lib = C.CDLL(p)
    vp, i32, i64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
    PC, PS, PR, PI = C.POINTER(kvc_cache), C.POINTER(kvc_state), C.POINTER(kvc_rope), C.POINTER(kvc_item)
    lib.kvc_apply.argtypes = [PC, PS, i32, PR, PC, vp]
    lib.kvc_chain.argtypes = [PC, i32, C.POINTER(i32), PS, PR, PC, vp]
    lib.kvc_chain_fused.argtypes = [PC, i32, C.POINTER(i32), PS, PR, PC, vp, sz, vp]
    lib.kvc_chain_workspace_bytes.argtypes = [PC, i32]
    lib.kvc_chain_workspace_bytes.restype = sz
    lib.kvc_state_update.argtypes = [PC, PC, i32, PR, PS, i32, vp, sz, vp]
    lib.kvc_state_update_noalloc.argtypes = [PC, PC, i32, PR, PS, i32, vp]
    lib.kvc_selftest_wait_expiry.argtypes = [C.c_double, C.POINTER(i32), vp]
    PSeg = C.POINTER(kvc_segments)
    lib.kvc_apply_segmented.argtypes = [PC, PS, PSeg, PR, PC, vp]
    lib.kvc_state_update_segmented.argtypes = [PC, PC, PSeg, PR, PS, i32, vp, sz, vp]
    lib.kvc_state_update_check.argtypes = [PC, PC, i32, PR, PS, i32]
    lib.kvc_state_update_chain.argtypes = [PC, i32, C.POINTER(i32), PR, PS, i32, vp, sz, vp]
    lib.kvc_chain_update_workspace_bytes.argtypes = [PC, i32, PS, i32]
    lib.kvc_chain_update_workspace_bytes.restype = sz
    lib.kvc_chain_update_edge_stride.argtypes = [PC, PS, i32]
    lib.kvc_chain_update_edge_stride.restype = sz
    lib.kvc_state_update_noalloc.restype = C.c_int
    lib.kvc_workspace_bytes.argtypes = [PC, PS, i32]
    lib.kvc_workspace_bytes.restype = sz
    lib.kvc_apply_batch.argtypes = [PI, i32, PR, vp, sz, vp, vp]
    lib.kvc_batch_workspace_bytes.argtypes = [i32]
    lib.kvc_batch_workspace_bytes.restype = sz
    lib.kvc_apply_multi.argtypes = [PC, PS, i32, vp, vp, i32, PR, PC, vp, sz, vp]
    lib.kvc_multi_workspace_bytes.argtypes = [PC, PS, i32]
    lib.kvc_multi_workspace_bytes.restype = sz
    lib.kvc_effective_rank.argtypes = [vp, i32, i32, C.c_double, vp, vp]
    lib.kvc_fit_eigenvalues.argtypes = [PC, vp]
    lib.kvc_fit_eigenvalues.restype = vp
    lib.kvc_fit_solver.argtypes = [PC, vp]
    lib.kvc_fit_solver.restype = vp
    lib.kvc_group_fit_eigenvalues.argtypes = [PC, vp]
    lib.kvc_group_fit_eigenvalues.restype = vp
    lib.kvc_group_fit_solver.argtypes = [PC, vp]
    lib.kvc_group_fit_solver.restype = vp
    lib.kvc_state_realign.argtypes = [PS, i32, i32, i32, i32, PR, vp, vp]
    lib.kvc_token_weights.argtypes = [PC, i32, PS, C.POINTER(i32), i32, PR, C.c_double, vp, vp, vp, sz, vp]
    lib.kvc_token_weights_workspace_bytes.argtypes = [PC, i32]
    lib.kvc_token_weights_workspace_bytes.restype = sz
    lib.kvc_gate_distance.argtypes = [PC, PS, i32, i32, vp, vp]
    lib.kvc_gate_weights.argtypes = [vp, i32, C.c_double, vp, vp, vp]
    # the calls of a serving step: descriptors go in as addresses (no pointer objects are made per call)
    lib.kvc_quantize.argtypes = lib.kvc_dequantize.argtypes = [vp, vp, vp]
    lib.kvc_append.argtypes = lib.kvc_append_q8.argtypes = [vp, vp, vp, i32, vp, vp]
    lib.kvc_attend.argtypes = lib.kvc_attend_q8.argtypes = [vp, vp, vp, i32, C.c_double, i32, vp, vp, vp, sz, vp]
    lib.kvc_attend_workspace_bytes.argtypes = [vp, i32, i32, i32]
    lib.kvc_attend_workspace_bytes.restype = sz
    lib.kvc_tree_build.argtypes = [vp, vp, vp]
    lib.kvc_append_rotated.argtypes = lib.kvc_append_rotated_q8.argtypes = [vp, vp, vp, vp, vp, vp, i32, vp, vp]
    lib.kvc_attend_tree.argtypes = lib.kvc_attend_tree_q8.argtypes = [vp, vp, vp, vp, i32, C.c_double, vp, vp, vp, sz, vp]
    lib.kvc_verify.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, i32, vp, vp, vp]
    lib.kvc_keep.argtypes = lib.kvc_keep_q8.argtypes = [vp, vp, i32, vp, vp, vp, vp]
    lib.kvc_block_append_rotated.argtypes = lib.kvc_block_attend_tree.argtypes = lib.kvc_block_verify.argtypes = lib.kvc_block_keep.argtypes = [vp]
    lib.kvc_status_poll.argtypes = [C.POINTER(C.c_uint32)]
    lib.kvc_status_reset.argtypes = []
    lib.kvc_set_path.argtypes = [i32]
    lib.kvc_last_path.argtypes = []
    lib.kvc_apply_bytes.argtypes = [PC, PS]
    lib.kvc_apply_bytes.restype = i64
    lib.kvc_update_bytes.argtypes = [PC, PS, i32, i32]
    lib.kvc_update_bytes.restype = i64
    lib.kvc_strerror.argtypes = [C.c_int]
    lib.kvc_strerror.restype = C.c_char_p
    lib.kvc_version.argtypes = []
    lib.kvc_version.restype = C.c_char_p
    for name in ("kvc_apply", "kvc_chain", "kvc_state_update", "kvc_apply_batch", "kvc_status_poll",
                 "kvc_status_reset", "kvc_set_path", "kvc_last_path"):
        getattr(lib, name).restype = C.c_int
    if path is None:
        _lib = lib
    return lib


def strerror(code: int) -> str:
    return load().kvc_strerror(code).decode()


def version() -> str:
    return load().kvc_version().decode()


# ---- descriptors over torch tensors ------------------------------------------------


class _Described:
    """Base of the caches: setting an attribute drops the descriptor kept between calls."""

    def __setattr__(self, name, value):
        self.__dict__.pop("_made", None)
        object.__setattr__(self, name, value)

    def __getstate__(self):                       # copies and pickles make a descriptor of their own
        return {k: v for k, v in self.__dict__.items() if k != "_made"}


class Cache(_Described):
    """A cache descriptor over torch tensors (which it keeps alive).

    contiguous: ``k``, ``v`` bf16 [L, H, T, d]; ``token_major=True``: [L, T, H, d] (each token with all its
                heads), described to the library through the strides.
    paged:      ``k``, ``v`` bf16 pools [L, P, H, page, d], ``page_table`` int32
                [ceil(T/page)], ``T`` the logical length.  ``token_major=True``: the pools
                are [L, P, page, H, d] (a page holds its tokens one after the other, each
                with all heads), described to the library through the strides.
    """

    def __init__(self, k: torch.Tensor, v: torch.Tensor, T: Optional[int] = None,
                 page_table: Optional[torch.Tensor] = None, token_major: bool = False):
        assert k.dtype == torch.bfloat16 and v.dtype == torch.bfloat16
        assert k.is_contiguous() and v.is_contiguous() and k.shape == v.shape
        self.k, self.v, self.page_table = k, v, page_table
        self.token_major = bool(token_major)
        if page_table is None:
            if token_major:
                self.L, self.T, self.H, self.d = (int(x) for x in k.shape)
            else:
                self.L, self.H, self.T, self.d = (int(x) for x in k.shape)
            self.page, self.P = 0, 0
        else:
            assert page_table.dtype == torch.int32 and page_table.is_contiguous() and T is not None
            if token_major:
                self.L, self.P, self.page, self.H, self.d = (int(x) for x in k.shape)
            else:
                self.L, self.P, self.H, self.page, self.d = (int(x) for x in k.shape)
            self.T = int(T)

    def struct(self) -> kvc_cache:
        s = kvc_cache()
        s.k, s.v = self.k.data_ptr(), self.v.data_ptr()
        s.L, s.H, s.T, s.d = self.L, self.H, self.T, self.d
        if self.page_table is None:
            s.layout = KVC_CONTIG
            if self.token_major:
                s.s_tok, s.s_head = self.H * self.d, self.d
                s.s_layer = self.T * self.H * self.d
        else:
            s.layout = KVC_PAGED
            s.page_size, s.n_phys_pages = self.page, self.P
            s.page_table = self.page_table.data_ptr()
            if self.token_major:
                s.s_tok, s.s_head = self.H * self.d, self.d
                s.s_page = self.page * self.H * self.d
                s.s_layer = self.P * s.s_page
        return s

    def empty_like(self, page_table: Optional[torch.Tensor] = None, fill: Optional[float] = None) -> "Cache":
        mk = (lambda t: torch.empty_like(t)) if fill is None else (lambda t: torch.full_like(t, fill))
        if self.page_table is None:
            return Cache(mk(self.k), mk(self.v), token_major=self.token_major)
        return Cache(mk(self.k), mk(self.v), T=self.T,
                     page_table=self.page_table if page_table is None else page_table, token_major=self.token_major)

    def nbytes(self) -> int:
        return self.k.numel() * 2 + self.v.numel() * 2

    @staticmethod
    def pool(k: torch.Tensor, v: torch.Tensor, token_major: bool = False) -> "Cache":
        """A paged pool without a table of its own: its pages belong to requests (:class:`Requests`)."""
        return Cache(k, v, T=0, page_table=torch.empty(0, dtype=torch.int32, device=k.device), token_major=token_major)


class QCache(_Described):
    """A cache held in 8 bits: ``k``, ``v`` float8_e4m3fn codes in the shapes of :class:`Cache`, ``scale_k``, ``scale_v``
    uint8 exponents of the same shapes without the channel axis (value = code * 2^(exponent - 127))."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, scale_k: torch.Tensor, scale_v: torch.Tensor, T: Optional[int] = None,
                 page_table: Optional[torch.Tensor] = None, token_major: bool = False):
        assert k.dtype == torch.float8_e4m3fn and v.dtype == torch.float8_e4m3fn
        assert k.is_contiguous() and v.is_contiguous() and k.shape == v.shape
        for e in (scale_k, scale_v):
            assert e.dtype == torch.uint8 and e.is_contiguous() and e.shape == k.shape[:-1]
        self.k, self.v, self.scale_k, self.scale_v = k, v, scale_k, scale_v
        self.page_table, self.token_major = page_table, bool(token_major)
        if page_table is None:
            self.L, self.T, self.H, self.d = (int(x) for x in (k.shape if token_major else k.transpose(1, 2).shape))
            self.page, self.P = 0, 0
        else:
            assert page_table.dtype == torch.int32 and page_table.is_contiguous() and T is not None
            self.L, self.P, self.page, self.H, self.d = (int(x) for x in (k.shape if token_major else k.transpose(2, 3).shape))
            self.T = int(T)

    @staticmethod
    def pool(k, v, scale_k, scale_v, token_major: bool = False) -> "QCache":
        """A paged pool without a table of its own: its pages belong to requests (:class:`Requests`)."""
        return QCache(k, v, scale_k, scale_v, T=0, page_table=torch.empty(0, dtype=torch.int32, device=k.device),
                      token_major=token_major)

    @staticmethod
    def like(c: Cache) -> "QCache":
        """An empty 8-bit cache of ``c``'s geometry (and page table)."""
        code = lambda t: torch.zeros(t.shape, dtype=torch.float8_e4m3fn, device=t.device)
        exp = lambda t: torch.zeros(t.shape[:-1], dtype=torch.uint8, device=t.device)
        return QCache(code(c.k), code(c.v), exp(c.k), exp(c.v), T=None if c.page_table is None else c.T,
                      page_table=c.page_table, token_major=c.token_major)

    def struct(self) -> kvc_qcache:
        q = kvc_qcache()
        s = q.codes
        s.k, s.v = self.k.data_ptr(), self.v.data_ptr()
        s.L, s.H, s.T, s.d = self.L, self.H, self.T, self.d
        q.scale_k, q.scale_v = self.scale_k.data_ptr(), self.scale_v.data_ptr()
        if self.page_table is not None:
            s.layout, s.page_size, s.n_phys_pages, s.page_table = KVC_PAGED, self.page, self.P, self.page_table.data_ptr()
        if self.token_major:
            rows = self.T if self.page_table is None else self.page
            s.s_tok, s.s_head, q.e_tok, q.e_head = self.H * self.d, self.d, self.H, 1
            if self.page_table is None:
                s.s_layer, q.e_layer = rows * s.s_tok, rows * self.H
            else:
                s.s_page, q.e_page = rows * s.s_tok, rows * self.H
                s.s_layer, q.e_layer = self.P * s.s_page, self.P * q.e_page
        return q

    def nbytes(self) -> int:
        return 2 * (self.k.numel() + self.scale_k.numel())


class Requests:
    """A serving step's requests: ``q_begin`` int32 [n+1], ``kv_len`` int32 [n] and ``page_table`` int32 [n, pages] on the
    GPU (None: every request reads the cache's own table or rows), and host bounds on their values.  Fixed once made: the
    tensors' contents may change from step to step, the tensors and the bounds not."""

    def __init__(self, q_begin: torch.Tensor, kv_len: torch.Tensor, max_q: int, max_kv: int, page_table: Optional[torch.Tensor] = None):
        assert q_begin.dtype == kv_len.dtype == torch.int32 and q_begin.is_contiguous() and kv_len.is_contiguous()
        assert q_begin.numel() == kv_len.numel() + 1
        stride = 0
        if page_table is not None:
            assert page_table.dtype == torch.int32 and page_table.dim() == 2 and page_table.shape[0] == kv_len.numel()
            assert page_table.shape[1] <= 1 or page_table.stride(1) == 1
            stride = int(page_table.stride(0)) if kv_len.numel() > 1 else int(page_table.shape[1])
            assert stride >= int(page_table.shape[1])
            assert max_kv >= 0
        made = kvc_requests(kv_len.numel(), int(max_q), int(max_kv), stride, q_begin.data_ptr(), kv_len.data_ptr(),
                            0 if page_table is None else page_table.data_ptr())
        devs = {t.get_device() for t in (q_begin, kv_len, page_table) if t is not None}
        self.__dict__.update(q_begin=q_begin, kv_len=kv_len, page_table=page_table, n=int(kv_len.numel()), max_q=int(max_q),
                             max_kv=int(max_kv), _pages=0 if page_table is None else int(page_table.shape[1]), _struct=made,
                             _at=C.addressof(made), _dev=devs.pop() if len(devs) == 1 else -1)

    def __setattr__(self, name, value):
        raise AttributeError(f"Requests.{name} is fixed; write into its tensors, or make another Requests")

    def __reduce__(self):
        return Requests, (self.q_begin, self.kv_len, self.max_q, self.max_kv, self.page_table)

    def struct(self) -> kvc_requests:
        return self._struct


class _Fixed:
    """Base of the descriptors of device lists: the tensors' contents may change from step to step, the tensors not."""

    def __setattr__(self, name, value):
        raise AttributeError(f"{type(self).__name__}.{name} is fixed; write into its tensors, or make another {type(self).__name__}")


def _list(t, what: str, dtype=torch.int32) -> int:
    """Address of a contiguous device list."""
    if isinstance(t, torch.Tensor) and t.dtype is dtype and t.is_contiguous():
        return t.data_ptr()
    raise KvcError(KVC_E_INVALID_ARG, f"{what}: contiguous {dtype} expected")


def _device_of(*tensors) -> int:
    devs = {t.get_device() for t in tensors if t is not None}
    return devs.pop() if len(devs) == 1 else -1


class Tree(_Fixed):
    """A step's drafted tokens: ``parent`` int32 [rows] (place of the new token a row continues within its request, -1: the
    cache), ``mask`` int32 [rows, words] (32 new tokens a word) and ``depth`` int32 [rows], which :func:`kvc_tree_build`
    fills; all on the GPU.  ``max_q``: bound on the new tokens of a request, as in :class:`Requests`."""

    def __init__(self, parent: torch.Tensor, max_q: int, mask: Optional[torch.Tensor] = None, depth: Optional[torch.Tensor] = None):
        _list(parent, "parent")
        rows, words = int(parent.numel()), max(1, (int(max_q) + 31) // 32)
        if mask is None:
            mask = torch.zeros(rows, words, dtype=torch.int32, device=parent.device)
        if depth is None:
            depth = torch.zeros(rows, dtype=torch.int32, device=parent.device)
        _list(mask, "mask"), _list(depth, "depth")
        if parent.dim() != 1 or mask.dim() != 2 or mask.shape[0] != rows or mask.shape[1] < words or depth.shape != parent.shape:
            raise KvcError(KVC_E_SHAPE, f"parent [rows], mask [rows, {words} or more] and depth [rows] expected")
        made = kvc_tree(int(mask.shape[1]), rows, parent.data_ptr(), mask.data_ptr(), depth.data_ptr())
        self.__dict__.update(parent=parent, mask=mask, depth=depth, max_q=int(max_q), _struct=made, _at=C.addressof(made),
                             _dev=_device_of(parent, mask, depth))

    def __reduce__(self):
        return Tree, (self.parent, self.max_q, self.mask, self.depth)

    def struct(self) -> kvc_tree:
        return self._struct


class State:
    """Rank-r state over torch tensors.  Per (layer, head): coeff fp32 [L,H,n_cov,r], basis fp32|bf16
    [L,H,r,d].  Per layer (``grouping=KVC_GROUP_LAYER``): coeff [L,n_cov,r], basis [L,r,H*d]."""

    def __init__(self, coeff_k, coeff_v, basis_k, basis_v, n_cov: Optional[int] = None, grouping: int = KVC_GROUP_HEAD):
        self.coeff_k, self.coeff_v, self.basis_k, self.basis_v = coeff_k, coeff_v, basis_k, basis_v
        self.grouping = int(grouping)
        g = self.grouping == KVC_GROUP_LAYER
        self.r = 0 if basis_k is None else int(basis_k.shape[1 if g else 2])
        self.n_cov = (0 if coeff_k is None else int(coeff_k.shape[1 if g else 2])) if n_cov is None else int(n_cov)
        if self.r > 0:
            assert basis_k.is_contiguous() and basis_v.is_contiguous() and basis_k.dtype == basis_v.dtype
            assert basis_k.dtype in (torch.float32, torch.bfloat16)
        if self.r > 0 and self.n_cov > 0:
            assert coeff_k.dtype == torch.float32 and coeff_v.dtype == torch.float32
            assert coeff_k.is_contiguous() and coeff_v.is_contiguous()
            assert int(coeff_k.shape[-2]) == self.n_cov and int(coeff_k.shape[-1]) == self.r

    @staticmethod
    def empty() -> "State":
        return State(None, None, None, None, n_cov=0)

    @staticmethod
    def values_only(coeff_v, basis_v) -> "State":
        """Value factors alone (what the reliability gate reads); the key pointers are NULL."""
        s = State.__new__(State)
        s.coeff_k = s.basis_k = None
        s.coeff_v, s.basis_v = coeff_v, basis_v
        s.r, s.n_cov = int(basis_v.shape[2]), int(coeff_v.shape[2])
        assert coeff_v.dtype == torch.float32 and coeff_v.is_contiguous() and basis_v.is_contiguous()
        assert basis_v.dtype in (torch.float32, torch.bfloat16) and int(coeff_v.shape[3]) == s.r
        return s

    # ---- a state as one self-describing blob (header, coefficients, bases): checkpoint / resume of a profiled
    # correction, and the way to keep a failing case.  Host-side plumbing only.
    _BLOB_MAGIC = b"KVCSTATE"

    def dump(self) -> bytes:
        import struct as _st
        parts, meta = [], []
        for t in (self.coeff_k, self.coeff_v, self.basis_k, self.basis_v):
            if t is None:
                meta.append((0, 0, ()))
                continue
            c = t.detach().cpu().contiguous()
            raw = c.view(torch.int16).numpy().tobytes() if c.dtype == torch.bfloat16 else c.numpy().tobytes()
            meta.append((1, 2 if c.dtype == torch.bfloat16 else 4, tuple(int(x) for x in c.shape)))
            parts.append(raw)
        head = self._BLOB_MAGIC + _st.pack("<5i", 1, self.r, self.n_cov, getattr(self, "grouping", KVC_GROUP_HEAD), len(meta))
        for present, esize, shape in meta:
            head += _st.pack("<3i", present, esize, len(shape)) + _st.pack("<%dq" % len(shape), *shape)
        return head + b"".join(parts)

    @staticmethod
    def load(blob: bytes, device="cpu") -> "State":
        import struct as _st
        import numpy as _np
        if blob[:8] != State._BLOB_MAGIC:
            raise ValueError("not a state blob")
        ver, r, n_cov, grouping, n = _st.unpack_from("<5i", blob, 8)
        if ver != 1 or n != 4:
            raise ValueError("unknown state blob version")
        off, meta = 8 + 20, []
        for _ in range(n):
            present, esize, nd = _st.unpack_from("<3i", blob, off)
            off += 12
            shape = _st.unpack_from("<%dq" % nd, blob, off)
            off += 8 * nd
            meta.append((present, esize, shape))
        ts = []
        for present, esize, shape in meta:
            if not present:
                ts.append(None)
                continue
            cnt = 1
            for x in shape:
                cnt *= x
            if esize == 2:
                a = _np.frombuffer(blob, dtype=_np.int16, count=cnt, offset=off).copy()
                t = torch.from_numpy(a).view(torch.bfloat16)
            else:
                a = _np.frombuffer(blob, dtype=_np.float32, count=cnt, offset=off).copy()
                t = torch.from_numpy(a)
            off += cnt * esize
            ts.append(t.reshape(shape).to(device))
        if off != len(blob):
            raise ValueError("state blob has trailing or missing bytes")
        if ts[0] is None and ts[2] is None and ts[3] is not None:
            return State.values_only(ts[1], ts[3])
        return State(ts[0], ts[1], ts[2], ts[3], n_cov=n_cov, grouping=grouping)

    def struct(self) -> kvc_state:
        s = kvc_state()
        ptr = lambda t: 0 if t is None else t.data_ptr()
        s.coeff_k, s.coeff_v, s.basis_k, s.basis_v = ptr(self.coeff_k), ptr(self.coeff_v), ptr(self.basis_k), ptr(self.basis_v)
        s.r, s.n_cov = self.r, self.n_cov
        s.grouping = getattr(self, "grouping", KVC_GROUP_HEAD)
        b = self.basis_k if self.basis_k is not None else self.basis_v
        s.basis_dtype = KVC_BF16 if (b is not None and b.dtype == torch.bfloat16) else KVC_F32
        return s


class Rope:
    def __init__(self, theta: float = 10000.0, pairing: int = KVC_ROPE_HALF, inv_freq: Optional[Sequence[float]] = None):
        self.theta, self.pairing = float(theta), int(pairing)
        self._tab = None if inv_freq is None else (C.c_double * len(inv_freq))(*[float(x) for x in inv_freq])

    def struct(self) -> kvc_rope:
        s = kvc_rope()
        s.theta, s.pairing = self.theta, self.pairing
        s.inv_freq = None if self._tab is None else C.cast(self._tab, C.c_void_p)
        return s


def scaled_frequencies(theta: float, rot_dim: int, factor: float = 1.0, original: Optional[int] = None, slow: float = 1.0,
                       fast: float = 32.0) -> List[float]:
    """Frequencies theta^(-2k / rot_dim) for contexts ``factor`` times longer than the model was trained on.  ``original``
    None: linearly, f / factor.  Otherwise by parts (YaRN, arXiv 2309.00071, section 3.2): a pair that turns at least ``fast``
    times over the ``original`` tokens keeps its frequency, one that turns at most ``slow`` times is divided by the factor,
    in between a mix linear in the number of turns."""
    import math
    f = [float(theta) ** (-2.0 * k / rot_dim) for k in range(rot_dim // 2)]
    if original is None:
        return [x / factor for x in f]
    keep = [min(1.0, max(0.0, (original * x / (2 * math.pi) - slow) / (fast - slow))) for x in f]
    return [x * (w + (1.0 - w) / factor) for x, w in zip(f, keep)]


class Rotary(_Fixed):
    """How new tokens are turned to their positions: ``rope`` (theta and pairing, or a table of rot_dim / 2 frequencies, see
    :func:`scaled_frequencies`), the number of channels that are rotated (``rot_dim``; None: all), a factor on them
    (``amplitude``), and on the GPU ``depth`` int32 [rows] (None: a chain) and ``pos_begin`` int32 [requests], the position of
    a cache's first token (None: 0).  Fixed once made."""

    def __init__(self, rope: Rope, rot_dim: Optional[int] = None, amplitude: float = 1.0, depth: Optional[torch.Tensor] = None,
                 pos_begin: Optional[torch.Tensor] = None):
        if not isinstance(rope, Rope):
            raise KvcError(KVC_E_INVALID_ARG, f"Rotary: Rope expected, not {type(rope).__name__}")
        if amplitude == 0.0:
            raise KvcError(KVC_E_INVALID_ARG, "Rotary: an amplitude of 0")
        for t in (depth, pos_begin):
            if t is not None:
                _list(t, "depth, pos_begin")
        made = kvc_rotary(rope.struct(), float(amplitude), int(rot_dim or 0), 0, None if depth is None else depth.data_ptr(),
                          None if pos_begin is None else pos_begin.data_ptr())
        # one table per width is worked out here, not at every call
        tables = {}
        table = None if rope._tab is None else list(rope._tab)
        self.__dict__.update(rope=rope, rot_dim=int(rot_dim or 0), amplitude=float(amplitude), depth=depth, pos_begin=pos_begin, _struct=made,
                             _at=C.addressof(made), _table=table, _tables=tables, _rows=-1 if depth is None else depth.numel(),
                             _requests=-1 if pos_begin is None else pos_begin.numel(), _dev=None if depth is None and pos_begin is None else _device_of(depth, pos_begin))

    def __reduce__(self):
        return Rotary, (self.rope, self.rot_dim or None, self.amplitude, self.depth, self.pos_begin)

    def struct(self) -> kvc_rotary:
        return self._struct

    def _for(self, d: int) -> int:
        """Address of the descriptor for heads of d channels."""
        made = self._tables.get(d)
        if made is None:
            rot = self.rot_dim or d
            if self._table is not None and 2 * len(self._table) != rot:
                raise KvcError(KVC_E_SHAPE, f"Rotary: {len(self._table)} frequencies for {rot} channels")
            f = self._table if self._table is not None else [self.rope.theta ** (-2.0 * k / rot) if self.rope.theta > 0 else float("nan") for k in range(rot // 2)]
            tab = (C.c_double * max(1, len(f)))(*f)
            s = kvc_rotary.from_buffer_copy(self._struct)
            s.rope.inv_freq = C.cast(tab, C.c_void_p)
            made = self._tables[d] = (C.addressof(s), s, tab)
        return made[0]


def _stream(stream) -> int:
    if stream is None:
        stream = torch.cuda.current_stream()
    return int(stream.cuda_stream) if hasattr(stream, "cuda_stream") else int(stream)


def _check(code: int, what: str):
    if code != 0:
        raise KvcError(code, what)


# ---- the C ABI, same names ---------------------------------------------------------


def kvc_apply(src: Cache, st: State, shift: int, rope: Rope, dst: Cache, stream=None) -> None:
    s, d, t, r = src.struct(), dst.struct(), st.struct(), rope.struct()
    _check(load().kvc_apply(C.byref(s), C.byref(t), int(shift), C.byref(r), C.byref(d), _stream(stream)), "kvc_apply")


def kvc_chain(agent0: Cache, prefix_len: Sequence[int], states: Sequence[State], rope: Rope, outs: Sequence[Cache],
              stream=None) -> None:
    n = len(prefix_len)
    a0, r = agent0.struct(), rope.struct()
    pl = (C.c_int32 * n)(*[int(x) for x in prefix_len])
    sts = (kvc_state * max(n - 1, 1))(*[s.struct() for s in states])
    os_ = (kvc_cache * max(n - 1, 1))(*[o.struct() for o in outs])
    _check(load().kvc_chain(C.byref(a0), n, pl, sts, C.byref(r), os_, _stream(stream)), "kvc_chain")


def kvc_chain_workspace_bytes(agent0: Cache, n_agents: int) -> int:
    a0 = agent0.struct()
    return int(load().kvc_chain_workspace_bytes(C.byref(a0), int(n_agents)))


def kvc_chain_fused(agent0: Cache, prefix_len: Sequence[int], states: Sequence[State], rope: Rope, outs: Sequence[Cache],
                    workspace: torch.Tensor, stream=None) -> None:
    """kvc_chain in one pass over agent 0's cache (same results bit for bit)."""
    n = len(prefix_len)
    a0, r = agent0.struct(), rope.struct()
    pl = (C.c_int32 * n)(*[int(x) for x in prefix_len])
    sts = (kvc_state * max(n - 1, 1))(*[s.struct() for s in states])
    os_ = (kvc_cache * max(n - 1, 1))(*[o.struct() for o in outs])
    _check(load().kvc_chain_fused(C.byref(a0), n, pl, sts, C.byref(r), os_, workspace.data_ptr(),
                                  workspace.numel() * workspace.element_size(), _stream(stream)), "kvc_chain_fused")


class Segments:
    """Piecewise-constant shifts over the token axis: segment j covers t_begin[j] .. t_begin[j+1]-1."""

    def __init__(self, t_begin: Sequence[int], shift: Sequence[int], coords: int = KVC_COORDS_TARGET):
        assert len(t_begin) == len(shift)
        self.t_begin, self.shift, self.coords = [int(x) for x in t_begin], [int(x) for x in shift], int(coords)
        self._tb = (C.c_int32 * len(self.t_begin))(*self.t_begin)
        self._sh = (C.c_int32 * len(self.shift))(*self.shift)

    def struct(self) -> kvc_segments:
        s = kvc_segments()
        s.n, s.t_begin, s.shift, s.coords = len(self.t_begin), self._tb, self._sh, self.coords
        return s


def kvc_apply_segmented(src: Cache, st: State, segs: Segments, rope: Rope, dst: Cache, stream=None) -> None:
    s, d, t, r, g = src.struct(), dst.struct(), st.struct(), rope.struct(), segs.struct()
    _check(load().kvc_apply_segmented(C.byref(s), C.byref(t), C.byref(g), C.byref(r), C.byref(d), _stream(stream)),
           "kvc_apply_segmented")


def kvc_state_update_segmented(src: Optional[Cache], tgt: Cache, segs: Segments, rope: Rope, st: State, mode: int,
                               workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    t, s, r, g = tgt.struct(), st.struct(), rope.struct(), segs.struct()
    sp = None
    if src is not None:
        ss = src.struct()
        sp = C.byref(ss)
    ws_ptr = 0 if workspace is None else workspace.data_ptr()
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(load().kvc_state_update_segmented(sp, C.byref(t), C.byref(g), C.byref(r), C.byref(s), int(mode), ws_ptr, ws_bytes,
                                             _stream(stream)), "kvc_state_update_segmented")


def kvc_selftest_wait_expiry(limit_ms: float = 1.0, stream=None):
    """(threads whose wait claimed success, abort flag, cycles waited) of a bounded wait made to run out."""
    res = (C.c_int32 * 3)()
    _check(load().kvc_selftest_wait_expiry(float(limit_ms), res, _stream(stream)), "kvc_selftest_wait_expiry")
    return int(res[0]), int(res[1]), int(res[2])


def kvc_chain_update_workspace_bytes(agents: Sequence[Cache], states: Sequence[State], mode: int) -> int:
    n = len(agents)
    ag = (kvc_cache * n)(*[a.struct() for a in agents])
    sts = (kvc_state * max(n - 1, 1))(*[s.struct() for s in states])
    return int(load().kvc_chain_update_workspace_bytes(ag, n, sts, int(mode)))


def kvc_chain_update_edge_stride(tgt: Cache, st: State, mode: int) -> int:
    t, s = tgt.struct(), st.struct()
    return int(load().kvc_chain_update_edge_stride(C.byref(t), C.byref(s), int(mode)))


def kvc_state_update_chain(agents: Sequence[Cache], prefix_len: Sequence[int], rope: Rope, states: Sequence[State],
                           mode: int, workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """The states of every edge agents[a-1] -> agents[a] in one call (all eigensolves in one launch)."""
    n = len(agents)
    ag = (kvc_cache * n)(*[a.struct() for a in agents])
    pl = (C.c_int32 * n)(*[int(x) for x in prefix_len])
    sts = (kvc_state * max(n - 1, 1))(*[s.struct() for s in states])
    r = rope.struct()
    ws_ptr = 0 if workspace is None else workspace.data_ptr()
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(load().kvc_state_update_chain(ag, n, pl, C.byref(r), sts, int(mode), ws_ptr, ws_bytes, _stream(stream)),
           "kvc_state_update_chain")


def kvc_workspace_bytes(tgt: Cache, st: State, mode: int) -> int:
    t, s = tgt.struct(), st.struct()
    return int(load().kvc_workspace_bytes(C.byref(t), C.byref(s), int(mode)))


def kvc_state_update(src: Optional[Cache], tgt: Cache, shift: int, rope: Rope, st: State, mode: int,
                     workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    t, s, r = tgt.struct(), st.struct(), rope.struct()
    sp = None
    if src is not None:
        ss = src.struct()
        sp = C.byref(ss)
    ws_ptr = 0 if workspace is None else workspace.data_ptr()
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(load().kvc_state_update(sp, C.byref(t), int(shift), C.byref(r), C.byref(s), int(mode), ws_ptr, ws_bytes,
                                   _stream(stream)), "kvc_state_update")


KVC_STATIC_SCRATCH_BYTES = 128 * (2 * 128 * 128 + 128) * 4 + 1024


def kvc_state_update_noalloc(src: Optional[Cache], tgt: Cache, shift: int, rope: Rope, st: State, mode: int,
                             stream=None) -> None:
    """kvc_state_update for callers that may not allocate device memory (an engine plugin
    working inside a pre-sized pool, a process whose memory is all committed to the KV
    pool): FIT-mode scratch is a fixed array inside the library, so there is no workspace
    argument.  Raises KvcError(-8) when the problem needs more than
    KVC_STATIC_SCRATCH_BYTES (L*H > 64 at d = 128).  Calls that may overlap on the GPU must
    be serialised by the caller: they share the one array."""
    t, s, r = tgt.struct(), st.struct(), rope.struct()
    sp = None
    if src is not None:
        ss = src.struct()
        sp = C.byref(ss)
    _check(load().kvc_state_update_noalloc(sp, C.byref(t), int(shift), C.byref(r), C.byref(s), int(mode),
                                           _stream(stream)), "kvc_state_update_noalloc")


class Item:
    """One work item of kvc_apply_batch; (t_begin, t_end) = (0, 0) means all rows of the caches."""

    def __init__(self, src: Cache, dst: Cache, st: State, shift: int, t_begin: int = 0, t_end: int = 0):
        self.src, self.dst, self.st, self.shift = src, dst, st, int(shift)
        self.t_begin, self.t_end = int(t_begin), int(t_end)


def kvc_batch_workspace_bytes(n_items: int) -> int:
    return int(load().kvc_batch_workspace_bytes(int(n_items)))


def kvc_apply_batch(items: Sequence[Item], rope: Rope, workspace: torch.Tensor, staging: torch.Tensor,
                    stream=None) -> None:
    n = len(items)
    arr = (kvc_item * max(n, 1))()
    for i, it in enumerate(items):
        arr[i].src, arr[i].dst, arr[i].st, arr[i].shift = it.src.struct(), it.dst.struct(), it.st.struct(), it.shift
        arr[i].t_begin, arr[i].t_end = getattr(it, "t_begin", 0), getattr(it, "t_end", 0)
    r = rope.struct()
    assert staging.device.type == "cpu" and staging.numel() * staging.element_size() >= kvc_batch_workspace_bytes(n)
    _check(load().kvc_apply_batch(arr, n, C.byref(r), workspace.data_ptr(),
                                  workspace.numel() * workspace.element_size(), staging.data_ptr(), _stream(stream)),
           "kvc_apply_batch")


KVC_MULTI_MAX_BLOCKS = 10


def kvc_multi_tpad(T: int) -> int:
    return (int(T) + 127) // 128 * 128


def _state_array(states: Sequence[State]):
    arr = (kvc_state * max(len(states), 1))()
    for i, a in enumerate(states):
        arr[i] = a.struct()
    return arr


def kvc_multi_workspace_bytes(src: Cache, deltas: Sequence[State]) -> int:
    c = src.struct()
    return int(load().kvc_multi_workspace_bytes(C.byref(c), _state_array(deltas), len(deltas)))


def kvc_apply_multi(src: Cache, deltas: Sequence[State], w_k: Optional[torch.Tensor], w_v: Optional[torch.Tensor],
                    shift: int, rope: Rope, dst: Cache, workspace: torch.Tensor, stream=None) -> None:
    """Eq. 8 with token-wise weights [n_anchors, kvc_multi_tpad(T)] fp32 (None: all ones)."""
    cs, cd, r = src.struct(), dst.struct(), rope.struct()
    for w in (w_k, w_v):
        assert w is None or (w.dtype == torch.float32 and w.is_cuda and w.is_contiguous()
                             and tuple(w.shape) == (len(deltas), kvc_multi_tpad(src.T)))
    ptr = lambda t: 0 if t is None else t.data_ptr()
    _check(load().kvc_apply_multi(C.byref(cs), _state_array(deltas), len(deltas), ptr(w_k), ptr(w_v), int(shift),
                                  C.byref(r), C.byref(cd), workspace.data_ptr(),
                                  workspace.numel() * workspace.element_size(), _stream(stream)), "kvc_apply_multi")


KVC_MAX_ANCHORS = 16


def kvc_effective_rank(tgt: Cache, workspace: torch.Tensor, energy: float = 0.9, stream=None) -> torch.Tensor:
    """Effective ranks int32 [L, H, 2] (K, V) from the eigenvalues a FIT update left in `workspace`."""
    c = tgt.struct()
    ev = load().kvc_fit_eigenvalues(C.byref(c), workspace.data_ptr())
    out = torch.empty(tgt.L, tgt.H, 2, dtype=torch.int32, device=workspace.device)
    _check(load().kvc_effective_rank(ev, tgt.L * tgt.H * 2, tgt.d, float(energy), out.data_ptr(), _stream(stream)),
           "kvc_effective_rank")
    return out


def kvc_fit_solver(tgt: Cache, workspace: torch.Tensor) -> torch.Tensor:
    """int32 [L, H, 2] view into the workspace of a KVC_FIT_FAST update: KVC_SOLVER_SUBSPACE (0) where
    the subspace solver served the matrix, else the reason the full eigensolver ran."""
    c = tgt.struct()
    p = load().kvc_fit_solver(C.byref(c), workspace.data_ptr())
    if not p:
        raise KvcError(KVC_E_INVALID_ARG, "kvc_fit_solver")
    off = p - workspace.data_ptr()
    n = tgt.L * tgt.H * 2
    return workspace.view(torch.uint8)[off: off + 4 * n].view(torch.int32).view(tgt.L, tgt.H, 2)


def kvc_group_fit_eigenvalues(tgt: Cache, workspace: torch.Tensor) -> torch.Tensor:
    """float32 [L, 2, H d] view into the workspace of a layer-grouped FIT update."""
    c = tgt.struct()
    p = load().kvc_group_fit_eigenvalues(C.byref(c), workspace.data_ptr())
    if not p:
        raise KvcError(KVC_E_INVALID_ARG, "kvc_group_fit_eigenvalues")
    off = p - workspace.data_ptr()
    n = tgt.L * 2 * tgt.H * tgt.d
    return workspace.view(torch.uint8)[off: off + 4 * n].view(torch.float32).view(tgt.L, 2, tgt.H * tgt.d)


def kvc_group_fit_solver(tgt: Cache, workspace: torch.Tensor) -> torch.Tensor:
    """int32 [L, 2] view into the workspace of a layer-grouped FIT update: 0 where the result was accepted."""
    c = tgt.struct()
    p = load().kvc_group_fit_solver(C.byref(c), workspace.data_ptr())
    if not p:
        raise KvcError(KVC_E_INVALID_ARG, "kvc_group_fit_solver")
    off = p - workspace.data_ptr()
    n = tgt.L * 2
    return workspace.view(torch.uint8)[off: off + 4 * n].view(torch.int32).view(tgt.L, 2)


def kvc_state_realign(st: State, shift: int, rope: Rope, out: Optional[torch.Tensor] = None, stream=None) -> State:
    """A state whose key correction is re-aligned by `shift` positions: basis_k rows rotated (into `out`,
    a new tensor by default; pass st.basis_k for in place); coefficients and value factors are shared."""
    if getattr(st, "grouping", KVC_GROUP_HEAD) == KVC_GROUP_LAYER:
        raise KvcError(KVC_E_UNSUPPORTED, "kvc_state_realign on a per-layer state: pass its geometry through the C call")
    L, H, r, d = (int(x) for x in st.basis_k.shape)
    out = torch.empty_like(st.basis_k) if out is None else out
    s, rp = st.struct(), rope.struct()
    _check(load().kvc_state_realign(C.byref(s), L, H, d, int(shift), C.byref(rp), out.data_ptr(), _stream(stream)),
           "kvc_state_realign")
    return State(st.coeff_k, st.coeff_v, out, st.basis_v, n_cov=st.n_cov)


def kvc_token_weights_workspace_bytes(src: Cache, n_anchors: int) -> int:
    c = src.struct()
    return int(load().kvc_token_weights_workspace_bytes(C.byref(c), int(n_anchors)))


def kvc_token_weights(src: Cache, src_pos: int, anchors: Sequence[State], anchor_pos: Sequence[int], rope: Rope,
                      w_k: torch.Tensor, w_v: torch.Tensor, workspace: torch.Tensor, temperature: float = 1.0,
                      stream=None) -> None:
    """App. A.3 token-wise weights [n_anchors, kvc_multi_tpad(T)] fp32 for keys and for values."""
    n = len(anchors)
    c, r = src.struct(), rope.struct()
    pos = (C.c_int32 * max(n, 1))(*[int(x) for x in anchor_pos])
    for w in (w_k, w_v):
        assert w.dtype == torch.float32 and w.is_cuda and w.is_contiguous() and tuple(w.shape) == (n, kvc_multi_tpad(src.T))
    _check(load().kvc_token_weights(C.byref(c), int(src_pos), _state_array(anchors), pos, n, C.byref(r), float(temperature),
                                    w_k.data_ptr(), w_v.data_ptr(), workspace.data_ptr(),
                                    workspace.numel() * workspace.element_size(), _stream(stream)), "kvc_token_weights")


def kvc_gate_distance(src: Cache, anchors: Sequence[State], k: int, dist_sq: torch.Tensor, stream=None) -> None:
    """Eq. 9, squared: dist_sq[v] (device float64 [len(anchors)]) for every anchor's value factors."""
    n = len(anchors)
    arr = (kvc_state * max(n, 1))()
    for i, a in enumerate(anchors):
        arr[i] = a.struct()
    c = src.struct()
    assert dist_sq.dtype == torch.float64 and dist_sq.is_cuda and dist_sq.numel() >= n
    _check(load().kvc_gate_distance(C.byref(c), arr, n, int(k), dist_sq.data_ptr(), _stream(stream)), "kvc_gate_distance")


def kvc_gate_weights(dist_sq: torch.Tensor, g: torch.Tensor, entropy: torch.Tensor, temperature: float = 1.0,
                     stream=None) -> None:
    """Eqs. 10-11 on the device: g = softmax(-sqrt(dist_sq)/T), entropy[0] = normalised entropy of g."""
    n = int(dist_sq.numel())
    assert dist_sq.dtype == g.dtype == entropy.dtype == torch.float64 and g.numel() >= n and entropy.numel() >= 1
    _check(load().kvc_gate_weights(dist_sq.data_ptr(), n, float(temperature), g.data_ptr(), entropy.data_ptr(),
                                   _stream(stream)), "kvc_gate_weights")


_HEADS = struct.Struct("@QiiQQ")      # kvc_heads


def _heads(t: torch.Tensor, d: int, what: str) -> bytes:
    """A kvc_heads over bf16 [rows, heads, d] with contiguous channels."""
    if not isinstance(t, torch.Tensor) or t.dtype is not torch.bfloat16 or t.dim() != 3:
        raise KvcError(KVC_E_INVALID_ARG, f"{what}: bf16 [rows, heads, d] expected")
    (rows, heads, dd), (s_row, s_head, s_ch) = t.shape, t.stride()
    if dd != d:
        raise KvcError(KVC_E_SHAPE, what)
    if s_ch != 1 or (rows > 1 and s_row == 0) or (heads > 1 and s_head == 0):
        raise KvcError(KVC_E_UNSUPPORTED, f"{what}: contiguous channels and no broadcast rows expected")
    return _HEADS.pack(t.data_ptr(), rows, heads, s_row if rows > 1 else 0, s_head if heads > 1 else 0)


def _fits(c, q8: bool, what: str) -> None:
    """The tensors hold what the descriptor will say they do, and the page table names a page for every token (attributes
    may have been set since the object was made)."""
    rows = c.L * c.H * (c.T if c.page_table is None else c.P * c.page)
    dtype = torch.float8_e4m3fn if q8 else torch.bfloat16
    for t, n, want in ((c.k, rows * c.d, dtype), (c.v, rows * c.d, dtype)) + (((c.scale_k, rows, torch.uint8), (c.scale_v, rows, torch.uint8)) if q8 else ()):
        if t.dtype is not want or not t.is_contiguous():
            raise KvcError(KVC_E_INVALID_ARG, f"{what}: contiguous {want} expected")
        if t.numel() < n:
            raise KvcError(KVC_E_SHAPE, f"{what}: a tensor of {t.numel()} elements for {n}")
    if c.page_table is not None:
        if c.page_table.dtype is not torch.int32 or not c.page_table.is_contiguous():
            raise KvcError(KVC_E_INVALID_ARG, f"{what}: contiguous int32 page table expected")
        if c.T > c.page_table.numel() * c.page:
            raise KvcError(KVC_E_SHAPE, f"{what}: {c.page_table.numel()} pages of {c.page} for {c.T} tokens")


def _desc(c, kind=None, what: str = "cache"):
    """(address of the descriptor of a Cache or QCache, its device, ..., its kvc_qcache or None): the structure is kept until
    an attribute of the object is set, its pointers are set at every call.  Addresses carry no type, so the class is
    checked here: `kind`, or either."""
    if not isinstance(c, _Described if kind is None else kind):
        raise KvcError(KVC_E_INVALID_ARG, f"{what}: a {'Cache or QCache' if kind is None else kind.__name__} expected, not {type(c).__name__}")
    made = c.__dict__.get("_made")
    if made is None:
        q8 = isinstance(c, QCache)
        _fits(c, q8, what)
        s = c.struct()
        devs = {t.get_device() for t in (c.k, c.v, c.page_table) + ((c.scale_k, c.scale_v) if q8 else ()) if t is not None}
        made = c.__dict__["_made"] = (C.addressof(s), devs.pop() if len(devs) == 1 else -1, s.codes if q8 else s, s if q8 else None)
    rows, q = made[2], made[3]
    rows.k, rows.v = c.k.data_ptr(), c.v.data_ptr()
    if c.page_table is not None:
        rows.page_table = c.page_table.data_ptr()
    if q is not None:
        q.scale_k, q.scale_v = c.scale_k.data_ptr(), c.scale_v.data_ptr()
    return made


def _here(what: str, stream, made, *tensors):
    """The stream to launch on; everything has to live on the current CUDA device, the one the library launches on."""
    cur = torch._C._cuda_getDevice() if torch.cuda.is_initialized() else -2
    for dev in made:
        if dev != cur:
            raise KvcError(KVC_E_INVALID_ARG, f"{what}: tensors on the current CUDA device expected")
    for t in tensors:
        if t is not None and t.get_device() != cur:
            raise KvcError(KVC_E_INVALID_ARG, f"{what}: tensors on the current CUDA device expected")
    return torch._C._cuda_getCurrentRawStream(cur) if stream is None else _stream(stream)


def _address(req: Requests, what: str) -> int:
    if not isinstance(req, Requests):
        raise KvcError(KVC_E_INVALID_ARG, f"{what}: Requests expected, not {type(req).__name__}")
    return req._at


def _holds(req: Requests, c, what: str) -> None:
    if req.page_table is not None and c.page_table is not None and req.max_kv > req._pages * c.page:
        raise KvcError(KVC_E_SHAPE, what)


def kvc_quantize(src: Cache, dst: QCache, stream=None) -> None:
    """dst = e4m3(src), one power-of-two scale per (layer, head, token)."""
    s, d = _desc(src, Cache, "kvc_quantize: src"), _desc(dst, QCache, "kvc_quantize: dst")
    st = _here("kvc_quantize", stream, (s[1], d[1]))
    _check(load().kvc_quantize(s[0], d[0], st), "kvc_quantize")


def kvc_dequantize(src: QCache, dst: Cache, stream=None) -> None:
    """dst = bf16(code * 2^(exponent - 127))."""
    s, d = _desc(src, QCache, "kvc_dequantize: src"), _desc(dst, Cache, "kvc_dequantize: dst")
    st = _here("kvc_dequantize", stream, (s[1], d[1]))
    _check(load().kvc_dequantize(s[0], d[0], st), "kvc_dequantize")


def kvc_append(req: Requests, k_new: torch.Tensor, v_new: torch.Tensor, cache, layer: int, stream=None) -> None:
    """Write the new tokens' rows [rows, H, d] into `layer` of a Cache, or quantised into a QCache."""
    at, c, k, v = _address(req, "kvc_append"), _desc(cache), _heads(k_new, cache.d, "k_new"), _heads(v_new, cache.d, "v_new")
    st = _here("kvc_append", stream, (c[1], req._dev), k_new, v_new)
    _holds(req, cache, "kvc_append")
    fn = load().kvc_append if c[3] is None else load().kvc_append_q8
    _check(fn(at, k, v, int(layer), c[0], st), "kvc_append")


def kvc_attend_workspace_bytes(req: Requests, cache, n_heads: int) -> int:
    return int(load().kvc_attend_workspace_bytes(_address(req, "kvc_attend_workspace_bytes"), int(n_heads), cache.H, cache.d))


def kvc_attend(req: Requests, q: torch.Tensor, cache, layer: int, out: torch.Tensor, workspace: Optional[torch.Tensor] = None,
               scale: Optional[float] = None, causal: bool = True, lse: Optional[torch.Tensor] = None, stream=None) -> None:
    """Attention of the new tokens' queries [rows, heads, d] over `layer` of a Cache or QCache (scale: 1 / sqrt(d))."""
    at, c, hq, ho = _address(req, "kvc_attend"), _desc(cache), _heads(q, cache.d, "q"), _heads(out, cache.d, "out")
    st = _here("kvc_attend", stream, (c[1], req._dev), q, out, workspace, lse)
    _holds(req, cache, "kvc_attend")
    if workspace is not None and not workspace.is_contiguous():
        raise KvcError(KVC_E_INVALID_ARG, "kvc_attend: a contiguous workspace expected")
    if lse is not None and (lse.dtype is not torch.float32 or not lse.is_contiguous() or lse.shape != q.shape[:2]):
        raise KvcError(KVC_E_INVALID_ARG, "kvc_attend: lse must be float32 [rows, heads]")
    fn = load().kvc_attend if c[3] is None else load().kvc_attend_q8
    _check(fn(at, hq, c[0], int(layer), cache.d ** -0.5 if scale is None else float(scale), bool(causal), ho,
              None if lse is None else lse.data_ptr(), None if workspace is None else workspace.data_ptr(),
              0 if workspace is None else workspace.numel() * workspace.element_size(), st), "kvc_attend")


def _pack(*args) -> bytes:
    """An argument block of the calls below (``csrc/marshal.cpp``).  The module takes this function's place at the first
    call; no Python stands in for it."""
    global _pack
    try:
        from . import _marshal
    except ImportError as e:
        raise RuntimeError("_marshal not found for this interpreter: build it with `python -m paper_2609_34060_b200.build`") from e
    _marshal.setup(KvcError, torch.bfloat16, torch.float32, torch.int32)
    _pack = _marshal.pack
    return _pack(*args)


def _tree(tree, what: str) -> int:
    if not isinstance(tree, Tree):
        raise KvcError(KVC_E_INVALID_ARG, f"{what}: Tree expected, not {type(tree).__name__}")
    return tree._at


def _describe(c):
    """A cache whose descriptor is there (made at its first use, dropped when an attribute of it is set)."""
    if not isinstance(c, _Described) or "_made" not in c.__dict__:
        _desc(c)
    return c


def kvc_tree_build(req: Requests, tree: Tree, stream=None) -> None:
    """Masks and depths of a step's drafted tokens from their parents."""
    at, t = _address(req, "kvc_tree_build"), _tree(tree, "kvc_tree_build")
    st = _here("kvc_tree_build", stream, (req._dev, tree._dev))
    _check(load().kvc_tree_build(at, t, st), "kvc_tree_build")


_ROTATED_NAMES, _TREE_NAMES = ("cache", "q", "q_out", "k_new", "v_new"), ("cache", "lse", "workspace", "q", "out")
_VERIFY_NAMES = ("target", "draft", "parent", "token", "u", "u_next", "kept", "n_kept", "next_token")
_KEEP_NAMES = ("kept", "n_kept", "cache", "kv_out")


def kvc_append_rotated(req: Requests, rotary: Rotary, k_new: torch.Tensor, v_new: torch.Tensor, cache, layer: int, q: Optional[torch.Tensor] = None,
                       q_out: Optional[torch.Tensor] = None, stream=None) -> None:
    """Keys of the new tokens [rows, H, d] turned to their positions and written, with their values, into `layer` of a Cache
    or QCache; queries [rows, heads, d] of the same rows turned beside them (`q_out` may be `q`)."""
    what = "kvc_append_rotated"
    if not isinstance(rotary, Rotary):
        raise KvcError(KVC_E_INVALID_ARG, f"{what}: Rotary expected, not {type(rotary).__name__}")
    if (q is None) != (q_out is None):
        raise KvcError(KVC_E_INVALID_ARG, f"{what}: q and q_out go together")
    at, dev = _address(req, what), req._dev
    _describe(cache)
    st = _here(what, stream, (dev,) if rotary._dev is None else (dev, rotary._dev))
    _holds(req, cache, what)
    block = _pack("PPCPHHHHiiii", _ROTATED_NAMES, dev, cache.d, 0, 0, at, rotary._for(cache.d), cache, st, q, q_out, k_new, v_new, layer, q is not None,
                  rotary._rows, rotary._requests)
    _check(load().kvc_block_append_rotated(block), what)


def kvc_attend_tree(req: Requests, tree: Tree, q: torch.Tensor, cache, layer: int, out: torch.Tensor, workspace: Optional[torch.Tensor] = None,
                    scale: Optional[float] = None, lse: Optional[torch.Tensor] = None, stream=None) -> None:
    """Attention of a tree of drafted tokens: every row sees its request's context and the new tokens of its mask.
    Workspace: kvc_attend_workspace_bytes."""
    what = "kvc_attend_tree"
    at, t, dev = _address(req, what), _tree(tree, what), req._dev
    _describe(cache)
    st = _here(what, stream, (dev, tree._dev))
    _holds(req, cache, what)
    block = _pack("PPCFAPPdHHP", _TREE_NAMES, dev, cache.d, 0, 0, at, t, cache, lse, workspace, 0 if workspace is None else workspace.nbytes, st,
                  cache.d ** -0.5 if scale is None else scale, q, out, layer)
    if lse is not None and lse.shape != q.shape[:2]:
        raise KvcError(KVC_E_INVALID_ARG, f"{what}: lse must be float32 [rows, heads]")
    _check(load().kvc_block_attend_tree(block), what)


def kvc_verify(req: Requests, parent: torch.Tensor, token: torch.Tensor, target: torch.Tensor, u: torch.Tensor, u_next: torch.Tensor,
               kept: torch.Tensor, n_kept: torch.Tensor, next_token: torch.Tensor, draft: Optional[torch.Tensor] = None, stream=None) -> None:
    """Which drafted tokens stay (`kept` int32 [n, max_q], `n_kept` int32 [n]) and the token behind them (`next_token` int32
    [n]), from the target's distributions float32 [rows, vocabulary], those the drafts were drawn from, siblings independently
    of one another (None: they were chosen), and uniform random numbers `u` [rows], `u_next` [n]."""
    what = "kvc_verify"
    at, dev = _address(req, what), req._dev
    block = _pack("PpprrfuKnnPP", _VERIFY_NAMES, dev, 0, req.n, req.max_q, at, target, draft, parent, token, u, u_next, kept, n_kept, next_token,
                  _here(what, stream, (dev,)), draft is not None)
    _check(load().kvc_block_verify(block), what)


def kvc_keep(req: Requests, kept: torch.Tensor, n_kept: torch.Tensor, cache, kv_out: Optional[torch.Tensor] = None, stream=None) -> None:
    """The rows of the accepted drafts moved together in every layer of a Cache or QCache; `kv_out` int32 [n]: the lengths
    behind the step."""
    what = "kvc_keep"
    at, dev = _address(req, what), req._dev
    _describe(cache)
    _holds(req, cache, what)
    block = _pack("PKnCnP", _KEEP_NAMES, dev, 0, req.n, req.max_q, at, kept, n_kept, cache, kv_out, _here(what, stream, (dev,)))
    _check(load().kvc_block_keep(block), what)


def kvc_status_poll() -> int:
    w = C.c_uint32(0)
    rc = load().kvc_status_poll(C.byref(w))
    if rc not in (0, -7):
        raise KvcError(rc, "kvc_status_poll")
    return int(w.value)


def kvc_status_reset() -> None:
    _check(load().kvc_status_reset(), "kvc_status_reset")


def kvc_set_path(path: int) -> None:
    _check(load().kvc_set_path(int(path)), "kvc_set_path")


def kvc_last_path() -> int:
    return int(load().kvc_last_path())


def kvc_apply_bytes(src: Cache, st: State) -> int:
    s, t = src.struct(), st.struct()
    return int(load().kvc_apply_bytes(C.byref(s), C.byref(t)))


def kvc_update_bytes(tgt: Cache, st: State, mode: int, has_src: bool = True) -> int:
    s, t = tgt.struct(), st.struct()
    return int(load().kvc_update_bytes(C.byref(s), C.byref(t), int(mode), int(bool(has_src))))
