"""Thin ctypes binding over libdyspec.so: argument marshalling only.

Every step of the path runs in the HIP kernels behind the C ABI declared in
``include/dyspec.h``; torch is used for device memory and the current stream.  There is no
CPU fallback: if the library is missing or fails to load, importing callers get an error.
"""
from __future__ import annotations

import contextlib
import ctypes
import os
import struct
from dataclasses import dataclass
from typing import Optional, Sequence

import numpy as np

from . import build as _build

F32, BF16, BF16_WAVE = 0, 1, 0x101
MAX_SEQ, MAX_NODES, MAX_BUILD_NODES, MAX_VOCAB = 64, 2048, 1024, 32768
PAGED_COUNTER_BYTES = 16384
WS_BUILD_TREE, WS_TREE_ATTN, WS_VERIFY = 0, 1, 2
EXPORTS = ("dyspec_init", "dyspec_mask_words", "dyspec_workspace_bytes", "dyspec_status_string",
           "dyspec_build_tree", "dyspec_build_tree_threshold", "dyspec_build_tree_threshold_workspace_bytes",
           "dyspec_dfs_reorder", "dyspec_tree_attn", "dyspec_tree_attn_static_scratch", "dyspec_tree_attn_layers",
           "dyspec_tree_attn_layers_workspace_bytes", "dyspec_verify", "dyspec_verify_bf16",
           "dyspec_kv_append", "dyspec_kv_keep", "dyspec_paged_attn", "dyspec_paged_attn_workspace_bytes", "dyspec_prompt_attn",
           "dyspec_paged_attn_scored", "dyspec_paged_attn_scored_workspace_bytes", "dyspec_prompt_attn_scored",
           "dyspec_page_plan", "dyspec_sample", "dyspec_filter_logits",
           "dyspec_probe_mfma_bf16", "dyspec_probe_clock", "dyspec_probe_hbm_read")


class DyspecError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} ({status})")


class _Batch(ctypes.Structure):
    _fields_ = [("n_seq", ctypes.c_int32),
                ("node_offset", ctypes.POINTER(ctypes.c_int32)),
                ("prefix_len", ctypes.POINTER(ctypes.c_int32)),
                ("kv_offset", ctypes.POINTER(ctypes.c_int64))]


class _Tree(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in
                ("parent", "token", "sib_rank", "first_child", "next_sibling", "depth")]


class _PagedKV(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("page_table", ctypes.c_void_p), ("n_pages", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("max_pages", ctypes.c_int32), ("table_stride", ctypes.c_int32), ("page_stride", ctypes.c_int64)]


class _Scores(ctypes.Structure):
    _fields_ = [("cap", ctypes.c_float), ("window", ctypes.c_int32), ("rel_pos", ctypes.c_void_p)]


class _PagePool(ctypes.Structure):
    _fields_ = [("ring", ctypes.c_void_p), ("state", ctypes.c_void_p), ("n_pages", ctypes.c_int32), ("page_size", ctypes.c_int32)]


_lib = None
_torch = None       # the module, once the library is loaded (an import statement in every call is a microsecond of each)


def load_library(path: Optional[str] = None) -> ctypes.CDLL:
    """Load libdyspec.so (building it first only when nothing is built)."""
    global _lib, _torch
    if _lib is not None and path is None:
        return _lib
    p = path or _build.LIB
    if not os.path.exists(p):
        _build.build(force=True)
    # torch brings its own copy of the HIP runtime; it has to be the one in the process before
    # this library is mapped, or the two would run on separate runtimes and every pointer torch
    # hands over would be foreign to the kernels' launches
    import torch
    _torch = torch
    lib = ctypes.CDLL(p)
    V, I32, U64, SZ, F = ctypes.c_void_p, ctypes.c_int32, ctypes.c_uint64, ctypes.c_size_t, ctypes.c_float
    PB, PT = ctypes.POINTER(_Batch), ctypes.POINTER(_Tree)
    lib.dyspec_init.restype = I32
    lib.dyspec_init.argtypes = []
    lib.dyspec_mask_words.restype = I32
    lib.dyspec_mask_words.argtypes = [PB]
    lib.dyspec_workspace_bytes.restype = SZ
    lib.dyspec_workspace_bytes.argtypes = [I32, PB, I32, I32, I32, I32]
    lib.dyspec_status_string.restype = ctypes.c_char_p
    lib.dyspec_status_string.argtypes = [I32]
    lib.dyspec_build_tree.restype = I32
    lib.dyspec_build_tree.argtypes = [V, I32, PB, ctypes.POINTER(F), U64, PT, V, V, V, V, SZ, V]
    lib.dyspec_build_tree_threshold.restype = I32
    lib.dyspec_build_tree_threshold.argtypes = [V, I32, PB, ctypes.POINTER(F), ctypes.POINTER(ctypes.c_double), U64, PT,
                                                V, V, V, ctypes.POINTER(I32), V, SZ, V]
    lib.dyspec_build_tree_threshold_workspace_bytes.restype = SZ
    lib.dyspec_build_tree_threshold_workspace_bytes.argtypes = [PB]
    lib.dyspec_tree_attn.restype = I32
    lib.dyspec_tree_attn.argtypes = [V, V, V, V, V, V, PB, I32, I32, I32, I32, F, V, V, SZ, V]
    lib.dyspec_tree_attn_static_scratch.restype = I32
    lib.dyspec_tree_attn_static_scratch.argtypes = [V, V, V, V, V, V, PB, I32, I32, I32, I32, F, V, V]
    lib.dyspec_tree_attn_layers.restype = I32
    lib.dyspec_tree_attn_layers.argtypes = [V, V, V, V, V, V, PB, I32, ctypes.c_int64, ctypes.c_int64, ctypes.c_int64,
                                            I32, I32, I32, I32, F, V, V, SZ, V]
    lib.dyspec_tree_attn_layers_workspace_bytes.restype = SZ
    lib.dyspec_tree_attn_layers_workspace_bytes.argtypes = [PB, I32, I32, I32, I32]
    lib.dyspec_verify.restype = I32
    lib.dyspec_verify.argtypes = [V, V, I32, PB, PT, ctypes.POINTER(F), ctypes.POINTER(F), U64, I32,
                                  V, V, V, V, V, V, V, SZ, V]
    lib.dyspec_verify_bf16.restype = I32
    lib.dyspec_verify_bf16.argtypes = lib.dyspec_verify.argtypes
    lib.dyspec_dfs_reorder.restype = I32
    lib.dyspec_dfs_reorder.argtypes = [PB, PT, PT, V, V, V]
    I64, PC = ctypes.c_int64, ctypes.POINTER(_PagedKV)
    lib.dyspec_kv_append.restype = I32
    lib.dyspec_kv_append.argtypes = [V, I64, V, I64, V, I64, PC, PB, V, V, I32, I32, I32, I32, I32, I32, V, V, V]
    lib.dyspec_kv_keep.restype = I32
    lib.dyspec_kv_keep.argtypes = [PC, I32, I64, PB, V, V, I32, I32, I32, V]
    lib.dyspec_paged_attn.restype = I32
    lib.dyspec_paged_attn.argtypes = [V, PC, PB, V, I32, I32, I32, I32, F, V, V, SZ, V]
    lib.dyspec_paged_attn_workspace_bytes.restype = SZ
    lib.dyspec_paged_attn_workspace_bytes.argtypes = [PB, I32, I32, I32, I32]
    lib.dyspec_prompt_attn.restype = I32
    lib.dyspec_prompt_attn.argtypes = [V, I64, V, I64, V, I64, PB, I32, I32, I32, I32, F, V, V]
    PS = ctypes.POINTER(_Scores)
    lib.dyspec_paged_attn_scored.restype = I32
    lib.dyspec_paged_attn_scored.argtypes = [V, PC, PB, V, I32, I32, I32, I32, F, PS, V, V, SZ, V]
    lib.dyspec_paged_attn_scored_workspace_bytes.restype = SZ
    lib.dyspec_paged_attn_scored_workspace_bytes.argtypes = [PB, I32, I32, I32, I32, PS]
    lib.dyspec_prompt_attn_scored.restype = I32
    lib.dyspec_prompt_attn_scored.argtypes = [V, I64, V, I64, V, I64, PB, I32, I32, I32, I32, F, PS, V, V]
    lib.dyspec_page_plan.restype = I32
    lib.dyspec_page_plan.argtypes = [ctypes.POINTER(_PagePool), V, I32, I32, V, V, I32, V, V, I64, V, V]
    lib.dyspec_sample.restype = I32
    lib.dyspec_sample.argtypes = [V, I32, I32, I64, PB, V, V, V, V, V, V, V, V, V]
    lib.dyspec_filter_logits.restype = I32
    lib.dyspec_filter_logits.argtypes = [V, I32, I32, I64, PB, V, V, V, V, V, I64, V]
    lib.dyspec_probe_mfma_bf16.restype = I32
    lib.dyspec_probe_mfma_bf16.argtypes = [I32, I32, ctypes.POINTER(ctypes.c_double), V, V]
    lib.dyspec_probe_clock.restype = I32
    lib.dyspec_probe_clock.argtypes = [I32, V, ctypes.POINTER(I32), V]
    lib.dyspec_probe_hbm_read.restype = I32
    lib.dyspec_probe_hbm_read.argtypes = [V, SZ, V, V]
    if path is None:
        _lib = lib
    return lib


def init() -> None:
    """dyspec_init on torch's current device: code loading and kernel attributes up front."""
    _check(load_library().dyspec_init(), "dyspec_init")


def status_string(status: int) -> str:
    return load_library().dyspec_status_string(status).decode()


@dataclass
class Batch:
    """Host description of a ragged batch (see dyspec_batch in include/dyspec.h)."""
    node_offset: np.ndarray      # int32 [n_seq+1]
    prefix_len: np.ndarray       # int32 [n_seq]
    kv_offset: np.ndarray        # int64 [n_seq+1]

    @staticmethod
    def from_sizes(n_nodes: Sequence[int], prefix_len: Optional[Sequence[int]] = None) -> "Batch":
        n_nodes = list(n_nodes)
        prefix_len = [0] * len(n_nodes) if prefix_len is None else list(prefix_len)
        no = np.zeros(len(n_nodes) + 1, dtype=np.int32)
        no[1:] = np.cumsum(n_nodes)
        kv = np.zeros(len(n_nodes) + 1, dtype=np.int64)
        kv[1:] = np.cumsum(prefix_len)
        return Batch(no, np.asarray(prefix_len, dtype=np.int32), kv)

    @property
    def n_seq(self) -> int:
        return int(self.prefix_len.shape[0])

    @property
    def total_nodes(self) -> int:
        return int(self.node_offset[-1])

    @property
    def total_prefix(self) -> int:
        return int(self.kv_offset[-1])

    def _memo(self) -> dict:
        """Per-content cache (C struct, mask words, workspace sizes): calls in a layer loop
        describe the same batch again and again."""
        key = (self.node_offset.tobytes(), self.prefix_len.tobytes(), self.kv_offset.tobytes())
        memo = self.__dict__.get("_memo_store")
        if memo is None or memo["key"] != key:
            memo = {"key": key}
            self.__dict__["_memo_store"] = memo
        return memo

    def _c(self, memo: Optional[dict] = None) -> _Batch:
        if memo is None:
            memo = self._memo()
        c = memo.get("c")
        if c is None:
            no = np.ascontiguousarray(self.node_offset, dtype=np.int32)
            pl = np.ascontiguousarray(self.prefix_len, dtype=np.int32)
            kv = np.ascontiguousarray(self.kv_offset, dtype=np.int64)
            c = _Batch(self.n_seq,
                       no.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)),
                       pl.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)),
                       kv.ctypes.data_as(ctypes.POINTER(ctypes.c_int64)))
            memo["c"], memo["keep"] = c, (no, pl, kv)          # the struct points into these copies
        return c

    def _mask_words(self, memo: dict) -> int:
        words = memo.get("mask_words")
        if words is None:
            words = memo["mask_words"] = int(load_library().dyspec_mask_words(ctypes.byref(self._c(memo))))
        return words

    @property
    def mask_words(self) -> int:
        return self._mask_words(self._memo())


@dataclass
class Tree:
    """Device-resident packed token trees (see dyspec_tree in include/dyspec.h)."""
    parent: "torch.Tensor"
    token: "torch.Tensor"
    sib_rank: "torch.Tensor"
    first_child: "torch.Tensor"
    next_sibling: "torch.Tensor"
    depth: "torch.Tensor"

    def _c(self) -> _Tree:
        return _Tree(_ptr(self.parent, "int32"), _ptr(self.token, "int32"), _ptr(self.sib_rank, "int32"),
                     _ptr(self.first_child, "int32"), _ptr(self.next_sibling, "int32"), _ptr(self.depth, "int32"))

    @staticmethod
    def empty(total_nodes: int, device) -> "Tree":
        """Room for total_nodes rows.  The six arrays lie in one allocation, each aligned as one of its own would be (512 bytes):
        whoever holds one of them holds the memory of all."""
        import torch
        rows = torch.empty((6, -(-total_nodes // 128) * 128), dtype=torch.int32, device=device)
        return Tree(*rows[:, :total_nodes].unbind(0))

    @staticmethod
    def _empty_c(total_nodes: int, device) -> "tuple[Tree, _Tree]":
        """empty() on a GPU, and its pointers: no need to look at arrays just made."""
        tree = Tree.empty(total_nodes, device)
        if not tree.parent.is_cuda:
            raise ValueError("device tensor required")
        first, step = tree.parent.data_ptr(), -(-total_nodes // 128) * 512
        return tree, _Tree(first, first + step, first + 2 * step, first + 3 * step, first + 4 * step, first + 5 * step)


_dtypes: dict = {}


def _dtype(name: str):
    t = _dtypes.get(name)
    if t is None:
        import torch
        t = _dtypes[name] = getattr(torch, name)
    return t


def _ptr(t, want: Optional[str] = None) -> int:
    if t is None:
        return 0
    if not t.is_cuda:
        raise ValueError("device tensor required")
    if not t.is_contiguous():
        raise ValueError("contiguous tensor required")
    if want is not None and t.dtype is not (_dtypes.get(want) or _dtype(want)):
        raise ValueError(f"expected {want}, got {t.dtype}")
    return t.data_ptr()


def _stream(stream=None) -> int:
    if stream is not None:
        return int(stream.cuda_stream)
    torch = _torch or __import__("torch")
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _temps(x, n_seq: int):
    """fp32 per sequence, as a C array: a number for all, or one each."""
    if type(x) is float:
        a = (ctypes.c_float * n_seq)(*([x] * n_seq))
        return a, a
    if (type(x) is list or type(x) is tuple) and len(x) == n_seq and all(type(v) is float for v in x):
        a = (ctypes.c_float * n_seq)(*x)
        return a, a
    a = np.ascontiguousarray(np.broadcast_to(np.asarray(x, dtype=np.float32), (n_seq,)))
    return a, a.ctypes.data_as(ctypes.POINTER(ctypes.c_float))


def _check(status: int, where: str) -> None:
    if status != 0:
        raise DyspecError(status, where)


@dataclass
class BuiltTrees:
    tree: Tree
    est_value: "torch.Tensor"      # fp32 [sum N]
    anc_mask: "torch.Tensor"       # int64 view of u64 [sum N, mask_words]
    n_built: "torch.Tensor"        # int32 [n_seq]; -1: the builder gave up waiting for a draw


def build_tree(draft_logits, batch: Batch, draft_temp, seed: int, stream=None, use_workspace: bool = True) -> BuiltTrees:
    """dyspec_build_tree: greedy token-tree construction (Algorithm 1) + ancestor mask.
    use_workspace=False passes no workspace (the slower form that recomputes row sums)."""
    lib = load_library()
    torch = _torch
    dev = draft_logits.device
    total, n_seq, V = batch.total_nodes, batch.n_seq, int(draft_logits.shape[1])
    if draft_logits.shape[0] != total:
        raise ValueError("draft_logits needs one row per tree node")
    memo = batch._memo()
    cb = batch._c(memo)
    tree, ct = Tree._empty_c(total, dev)
    est = torch.empty(total, dtype=torch.float32, device=dev)
    mask = torch.empty((total, batch._mask_words(memo)), dtype=torch.int64, device=dev)
    nb = torch.empty(n_seq, dtype=torch.int32, device=dev)
    tarr, tptr = _temps(draft_temp, n_seq)
    ws, ws_bytes = None, 0
    if use_workspace:
        wkey = ("ws_build", V)
        if wkey not in memo:
            memo[wkey] = int(lib.dyspec_workspace_bytes(WS_BUILD_TREE, ctypes.byref(cb), V, 0, 0, 0))
        ws_bytes = memo[wkey]
        if ws_bytes:
            ws = torch.empty(ws_bytes // 8, dtype=torch.float64, device=dev)
    st = lib.dyspec_build_tree(_ptr(draft_logits, "float32"), V, ctypes.byref(cb), tptr, ctypes.c_uint64(seed),
                               ctypes.byref(ct), est.data_ptr(), mask.data_ptr(), nb.data_ptr(),
                               ws.data_ptr() if ws is not None else None, ctypes.c_size_t(ws_bytes), _stream(stream))
    _check(st, "dyspec_build_tree")
    return BuiltTrees(tree, est, mask, nb)


def build_tree_threshold(draft_logits, batch: Batch, draft_temp, threshold, seed: int, stream=None):
    """dyspec_build_tree_threshold: level-by-level construction with a threshold (Algorithm 2)
    + ancestor mask.  Returns (BuiltTrees, levels expanded); the call waits for the tree."""
    import torch
    lib = load_library()
    dev = draft_logits.device
    total, V = batch.total_nodes, int(draft_logits.shape[1])
    if draft_logits.shape[0] != total:
        raise ValueError("draft_logits needs one row per tree node")
    tree = Tree.empty(total, dev)
    est = torch.empty(total, dtype=torch.float32, device=dev)
    mask = torch.empty((total, batch.mask_words), dtype=torch.int64, device=dev)
    nb = torch.empty(batch.n_seq, dtype=torch.int32, device=dev)
    cb, ct = batch._c(), tree._c()
    tarr, tptr = _temps(draft_temp, batch.n_seq)
    thr = np.ascontiguousarray(np.broadcast_to(np.asarray(threshold, dtype=np.float64), (batch.n_seq,)))
    ws_bytes = int(lib.dyspec_build_tree_threshold_workspace_bytes(ctypes.byref(cb)))
    ws = torch.empty(max(ws_bytes // 8, 1), dtype=torch.float64, device=dev)
    levels = ctypes.c_int32(0)
    st = lib.dyspec_build_tree_threshold(_ptr(draft_logits, "float32"), V, ctypes.byref(cb), tptr,
                                         thr.ctypes.data_as(ctypes.POINTER(ctypes.c_double)), ctypes.c_uint64(seed),
                                         ctypes.byref(ct), _ptr(est), _ptr(mask), _ptr(nb), ctypes.byref(levels),
                                         _ptr(ws), ctypes.c_size_t(ws_bytes), _stream(stream))
    _check(st, "dyspec_build_tree_threshold")
    return BuiltTrees(tree, est, mask, nb), int(levels.value)


@dataclass
class ReorderedTrees:
    tree: Tree
    order: "torch.Tensor"          # int32 [sum N]: order[offset + new] = old local index
    anc_mask: "torch.Tensor"       # int64 view of u64 [sum N, mask_words]

    def gather_index(self, batch: "Batch"):
        """Global row indices: tensor[gather_index] puts token-aligned rows into the new order."""
        import torch
        off = torch.from_numpy(np.repeat(batch.node_offset[:-1], np.diff(batch.node_offset)).astype(np.int64))
        return self.order.long() + off.to(self.order.device)


def dfs_reorder(tree: Tree, batch: Batch, stream=None) -> ReorderedTrees:
    """dyspec_dfs_reorder: rename every tree's nodes in depth-first order (block-sparsity friendly)."""
    lib = load_library()
    torch = _torch
    dev = tree.parent.device
    total, memo = batch.total_nodes, batch._memo()
    cb, ci = batch._c(memo), tree._c()
    out, co = Tree._empty_c(total, dev)
    order = torch.empty(total, dtype=torch.int32, device=dev)
    mask = torch.empty((total, batch._mask_words(memo)), dtype=torch.int64, device=dev)
    _check(lib.dyspec_dfs_reorder(ctypes.byref(cb), ctypes.byref(ci), ctypes.byref(co), order.data_ptr(),
                                  mask.data_ptr(), _stream(stream)), "dyspec_dfs_reorder")
    return ReorderedTrees(out, order, mask)


_scratch_cache = {}


def _scratch(device, nbytes: int):
    """A zero-filled device buffer of at least nbytes, kept between calls (calls on one stream run
    in order, so consecutive layers can share it).  Tree attention wants the head of its workspace
    zero at the first call and leaves it zero, so the buffer is cleared once, here."""
    import torch
    key = str(device)
    buf = _scratch_cache.get(key)
    if buf is None or buf.numel() * 4 < nbytes:
        buf = torch.zeros((nbytes + 3) // 4, dtype=torch.float32, device=device)
        _scratch_cache[key] = buf
    return buf


def tree_attn_form(batch: "Batch", n_q_heads: int, n_kv_heads: int, head_dim: int, layers: int = 1, use_workspace: bool = True):
    """What a bf16 tree_attn call (with `layers`, a tree_attn_layers call) is launched as: (waves of a workgroup of the kernel
    for short walks or 0 for the kernel for long ones, parts of the prefix, 1 if the tree has a part of its own).
    For tests and benchmarks that name the kernel they are about; not an entry point of the C interface."""
    lib = load_library()
    cb, form = batch._c(), (ctypes.c_int32 * 3)()
    nbytes = lib.dyspec_tree_attn_layers_workspace_bytes(ctypes.byref(cb), layers, n_q_heads, n_kv_heads, head_dim) if use_workspace else 0
    _check(lib.dyspec_tree_attn_form(ctypes.byref(cb), layers, n_q_heads, n_kv_heads, head_dim, ctypes.c_size_t(nbytes), form),
           "dyspec_tree_attn_form")
    return tuple(form)


class PreparedCall:
    """One library call with its arguments checked and marshalled once.  Calling the object issues
    the call again on the stream it was prepared for (the current one at that time unless given),
    with the same tensors: what a loop that repeats a call wants, e.g. a decode loop's layers,
    where the checks and conversions of the plain functions cost more host time per call than a
    short kernel runs.  The object keeps its tensors alive; `out` is what the plain function
    returns."""
    __slots__ = ("_fn", "_args", "_keep", "_where", "out")

    def __init__(self, fn, args, keep, where, out):
        self._fn, self._args, self._keep, self._where, self.out = fn, args, keep, where, out

    def __call__(self):
        st = self._fn(*self._args)
        if st != 0:
            raise DyspecError(st, self._where)
        return self.out


def tree_attn(q, k_prefix, v_prefix, k_tree, v_tree, anc_mask, batch: Batch, softmax_scale: float,
              out=None, dtype: Optional[int] = None, stream=None, use_workspace: bool = True,
              static_scratch: bool = False):
    """dyspec_tree_attn: one layer of tree-masked attention.  q/out [sum N, Hq, d].
    use_workspace=False passes no workspace (then the prefix is never split over workgroups).
    static_scratch=True calls dyspec_tree_attn_static_scratch instead (the library's own static
    array in place of a workspace; `out` must be given: this path allocates nothing)."""
    return tree_attn_call(q, k_prefix, v_prefix, k_tree, v_tree, anc_mask, batch, softmax_scale, out, dtype, stream,
                          use_workspace, static_scratch)()


def tree_attn_call(q, k_prefix, v_prefix, k_tree, v_tree, anc_mask, batch: Batch, softmax_scale: float,
                   out=None, dtype: Optional[int] = None, stream=None, use_workspace: bool = True,
                   static_scratch: bool = False) -> PreparedCall:
    """tree_attn's call, prepared: nothing is launched until the returned object is called."""
    lib = load_library()
    torch = _torch
    total, Hq, d = q.shape
    kt_shape, q_dtype = k_tree.shape, q.dtype
    Hkv = int(kt_shape[1])
    if dtype is None:
        dtype = BF16 if q_dtype is torch.bfloat16 else {torch.float32: F32}[q_dtype]
    if total != batch.total_nodes or kt_shape[0] != total or v_tree.shape != kt_shape:
        raise ValueError("q / k_tree / v_tree need one row per tree node")
    prefix = batch.total_prefix
    if prefix > 0:
        kp_shape = k_prefix.shape
        if kp_shape[0] < prefix or kp_shape[1] != Hkv or kp_shape[2] != d or v_prefix.shape != kp_shape:
            raise ValueError("prefix K/V shape does not match the batch")
    memo = batch._memo()
    mask_shape = anc_mask.shape
    if mask_shape[0] != total or mask_shape[1] != batch._mask_words(memo):
        raise ValueError("ancestor mask shape does not match the batch")
    for t in (k_prefix, v_prefix, k_tree, v_tree):
        if t is not None and t.dtype != q_dtype:
            raise ValueError("q, k, v must share a dtype")
    if out is None:
        if static_scratch:
            raise ValueError("static_scratch=True needs the caller's `out` tensor")
        out = torch.empty_like(q)
    cb = batch._c(memo)
    keep = (q, k_prefix, v_prefix, k_tree, v_tree, anc_mask, out, batch, cb)
    if static_scratch:
        args = (_ptr(q), _ptr(k_prefix), _ptr(v_prefix), _ptr(k_tree), _ptr(v_tree), _ptr(anc_mask, "int64"),
                ctypes.byref(cb), int(Hq), Hkv, int(d), int(dtype), ctypes.c_float(softmax_scale), _ptr(out), _stream(stream))
        return PreparedCall(lib.dyspec_tree_attn_static_scratch, args, keep, "dyspec_tree_attn_static_scratch", out)
    ws, ws_bytes = None, 0
    if use_workspace and dtype == BF16:
        wkey = ("ws_attn", int(Hq), Hkv, int(d))
        if wkey not in memo:
            memo[wkey] = int(lib.dyspec_workspace_bytes(WS_TREE_ATTN, ctypes.byref(cb), 0, int(Hq), Hkv, int(d)))
        ws_bytes = memo[wkey]
        if ws_bytes:
            ws = _scratch(q.device, ws_bytes)
    args = (_ptr(q), _ptr(k_prefix), _ptr(v_prefix), _ptr(k_tree), _ptr(v_tree), _ptr(anc_mask, "int64"),
            ctypes.byref(cb), int(Hq), Hkv, int(d), int(dtype), ctypes.c_float(softmax_scale), _ptr(out),
            _ptr(ws) if ws is not None else None, ctypes.c_size_t(ws_bytes), _stream(stream))
    return PreparedCall(lib.dyspec_tree_attn, args, keep + (ws,), "dyspec_tree_attn", out)


def tree_attn_layers(q, k_prefix, v_prefix, k_tree, v_tree, anc_mask, batch: Batch, softmax_scale: float,
                     out=None, dtype: Optional[int] = None, stream=None, use_workspace: bool = True):
    """dyspec_tree_attn_layers: tree-masked attention of L stacked layers in one call.
    q/out [L, sum N, Hq, d], k_prefix/v_prefix [L, kv rows, Hkv, d], k_tree/v_tree [L, sum N, Hkv, d];
    the leading dimension may be strided, the rest is dense."""
    import torch
    lib = load_library()
    L, total, Hq, d = q.shape
    Hkv = int(k_tree.shape[2])
    if dtype is None:
        dtype = {torch.float32: F32, torch.bfloat16: BF16}[q.dtype]
    if total != batch.total_nodes or tuple(k_tree.shape) != (L, total, Hkv, d) or v_tree.shape != k_tree.shape:
        raise ValueError("q / k_tree / v_tree need one row per tree node and layer")
    if batch.total_prefix > 0 and (k_prefix.shape[0] != L or k_prefix.shape[1] < batch.total_prefix or k_prefix.shape[2] != Hkv
                                   or k_prefix.shape[3] != d or v_prefix.shape != k_prefix.shape):
        raise ValueError("prefix K/V shape does not match the batch")
    if anc_mask.shape[0] != total or anc_mask.shape[1] != batch.mask_words:
        raise ValueError("ancestor mask shape does not match the batch")
    if out is None:
        out = torch.empty_like(q)
    for t in (q, out, k_prefix, v_prefix, k_tree, v_tree):
        if t is None:
            continue
        if t.dtype != q.dtype:
            raise ValueError("q, k, v, out must share a dtype")
        if not t.is_cuda or not t[0].is_contiguous():
            raise ValueError("device tensors with dense layers required")
    if out.stride(0) != q.stride(0) or (k_prefix is not None and v_prefix.stride(0) != k_prefix.stride(0)) \
            or v_tree.stride(0) != k_tree.stride(0):
        raise ValueError("q/out, k_prefix/v_prefix and k_tree/v_tree must share their layer strides")
    cb = batch._c()
    ws, ws_bytes = None, 0
    if use_workspace and dtype == BF16:
        ws_bytes = int(lib.dyspec_tree_attn_layers_workspace_bytes(ctypes.byref(cb), int(L), int(Hq), Hkv, int(d)))
        if ws_bytes:
            ws = _scratch(q.device, ws_bytes)
    kp_stride = int(k_prefix.stride(0)) if k_prefix is not None else 0
    base = lambda t: 0 if t is None else t.data_ptr()          # the layer dimension may be strided
    st = lib.dyspec_tree_attn_layers(base(q), base(k_prefix), base(v_prefix), base(k_tree), base(v_tree),
                                     _ptr(anc_mask, "int64"), ctypes.byref(cb), int(L), int(q.stride(0)), kp_stride,
                                     int(k_tree.stride(0)), int(Hq), Hkv, int(d), int(dtype),
                                     ctypes.c_float(softmax_scale), base(out), _ptr(ws) if ws is not None else None,
                                     ctypes.c_size_t(ws_bytes), _stream(stream))
    _check(st, "dyspec_tree_attn_layers")
    return out


@dataclass
class VerifyOutput:
    row_stats: "torch.Tensor"        # fp32 [sum N, 4]
    accept_ratio: "torch.Tensor"     # fp32 [sum N]; -1 / -2 mark children the walk did not test
    accepted_nodes: "torch.Tensor"   # int32 [sum N]
    n_accepted: "torch.Tensor"       # int32 [n_seq]
    final_token: "torch.Tensor"      # int32 [n_seq]
    min_margin: "torch.Tensor"       # fp32 [n_seq]

    @staticmethod
    def empty(batch: Batch, device) -> "VerifyOutput":
        import torch
        t, s = batch.total_nodes, batch.n_seq
        f = lambda *sh: torch.empty(sh, dtype=torch.float32, device=device)
        i = lambda *sh: torch.empty(sh, dtype=torch.int32, device=device)
        return VerifyOutput(f(t, 4), f(t), i(t), i(s), i(s), f(s))


def verify(draft_logits, target_logits, batch: Batch, tree: Tree, draft_temp, target_temp, seed: int,
           emit_bonus: bool = True, out: Optional[VerifyOutput] = None, stream=None) -> VerifyOutput:
    """dyspec_verify / dyspec_verify_bf16 (by the tables' dtype): per-row vocabulary softmax + tree
    rejection sampling (Algorithm 3)."""
    return verify_call(draft_logits, target_logits, batch, tree, draft_temp, target_temp, seed, emit_bonus, out, stream)()


def verify_call(draft_logits, target_logits, batch: Batch, tree: Tree, draft_temp, target_temp, seed: int,
                emit_bonus: bool = True, out: Optional[VerifyOutput] = None, stream=None) -> PreparedCall:
    """verify's call, prepared: nothing is launched until the returned object is called."""
    lib = load_library()
    total, n_seq, shape, dtype = batch.total_nodes, batch.n_seq, draft_logits.shape, draft_logits.dtype
    V = int(shape[1])
    if shape[0] != total or target_logits.shape != shape:
        raise ValueError("logit tables need one row per tree node")
    bf16 = dtype is _torch.bfloat16
    if target_logits.dtype != dtype or not (bf16 or dtype is _torch.float32):
        raise ValueError("logit tables must both be float32 or both be bfloat16")
    entry = lib.dyspec_verify_bf16 if bf16 else lib.dyspec_verify
    if out is None:
        out = VerifyOutput.empty(batch, draft_logits.device)
    cb, ct = batch._c(), tree._c()
    da, dp = _temps(draft_temp, n_seq)
    ta, tp = _temps(target_temp, n_seq)
    args = (_ptr(draft_logits), _ptr(target_logits), V, ctypes.byref(cb), ctypes.byref(ct), dp, tp,
            ctypes.c_uint64(seed), int(bool(emit_bonus)), _ptr(out.row_stats), _ptr(out.accept_ratio),
            _ptr(out.accepted_nodes), _ptr(out.n_accepted), _ptr(out.final_token), _ptr(out.min_margin), None, 0,
            _stream(stream))
    keep = (draft_logits, target_logits, batch, tree, cb, ct, da, ta, out)
    return PreparedCall(entry, args, keep, "dyspec_verify_bf16" if bf16 else "dyspec_verify", out)


# ---------------------------------------------------------------------------------------- the paged cache and prompts

@dataclass(frozen=True)
class PagedCache:
    """A pool of K/V pages and the sequences' page tables (see dyspec_paged_kv in include/dyspec.h).

    k, v        [n_pages, page_size, Hkv, d], or [L, n_pages, page_size, Hkv, d] for all layers of a model; rows dense in a
                page, pages (and layers) may be strided: halves of one [n_pages, 2, page_size, Hkv, d] pool will do
    page_table  int32 [n_seq or more, max_pages]; rows may be strided

    kv_append and paged_attn work on one layer (`layer(l)`: to be made once a layer, it costs more host time than a call), kv_keep on
    all at once."""
    k: "torch.Tensor"
    v: "torch.Tensor"
    page_table: "torch.Tensor"

    def __post_init__(self):
        k, v, table = self.k, self.v, self.page_table
        if k.dim() not in (4, 5) or v.shape != k.shape or v.dtype != k.dtype:
            raise ValueError("k and v need one shape ([layers,] pages, rows, heads, head_dim) and dtype")
        n_pages, page, Hkv, d = k.shape[-4:]
        if k.dim() == 5 and k.shape[0] == 0:
            raise ValueError("a cache of no layer")
        for t in (k, v):
            if not t.is_cuda:
                raise ValueError("device tensor required")
            if (d > 1 and t.stride(-1) != 1) or (Hkv > 1 and t.stride(-2) != d) or (page > 1 and t.stride(-3) != Hkv * d):
                raise ValueError("a page's rows must be dense")
        if (n_pages > 1 and k.stride(-4) != v.stride(-4)) or (k.dim() == 5 and k.shape[0] > 1 and k.stride(0) != v.stride(0)):
            raise ValueError("k and v must share their strides")
        if table.dim() != 2 or table.dtype is not _dtype("int32") or not table.is_cuda or (table.shape[1] > 1 and table.stride(1) != 1):
            raise ValueError("page_table must be an int32 device tensor [n_seq, max_pages]")
        if v.device != k.device or table.device != k.device:
            raise ValueError("k, v and page_table must share a device")
        columns = int(table.shape[1])
        c = _PagedKV(k.data_ptr(), v.data_ptr(), table.data_ptr(), int(n_pages), int(page), columns,
                     int(table.stride(0)) if table.shape[0] > 1 else columns, int(k.stride(-4)) if n_pages > 1 else int(page * Hkv * d))
        layers = int(k.shape[0]) if k.dim() == 5 else 0
        for name, value in dict(_c=c, _ref=ctypes.byref(c), _heads=(int(Hkv), int(d)), _code=_code(k.dtype), _torch_dtype=k.dtype,
                                _device=k.get_device(), _rows=int(table.shape[0]), _layers=layers,
                                _layer_stride=int(k.stride(0)) if layers > 1 else 0).items():
            object.__setattr__(self, name, value)

    def layer(self, index: int) -> "PagedCache":
        return PagedCache(self.k[index], self.v[index], self.page_table)


def _code(dtype) -> int:
    if dtype is not _dtype("bfloat16") and dtype is not _dtype("float32"):
        raise ValueError(f"float32 or bfloat16 expected, got {dtype}")
    return BF16 if dtype is _dtype("bfloat16") else F32


class DeviceCall(PreparedCall):
    """A PreparedCall that is issued on its tensors' device whichever device is current."""
    __slots__ = ("_device",)

    def __init__(self, fn, args, keep, where, out, device):
        super().__init__(fn, args, keep, where, out)
        self._device = device

    def __call__(self):
        _issue(self._fn, self._args, self._device, self._where)
        return self.out


class _Nothing(PreparedCall):
    """The call of a batch without a token: empty tensors have no address to hand over."""
    __slots__ = ()

    def __init__(self, out):
        super().__init__(None, (), (), "", out)

    def __call__(self):
        return self.out


def _issue(fn, args, device: int, where: str) -> None:
    if _torch._C._cuda_getDevice() == device:
        st = fn(*args)
    else:
        with _torch.cuda.device(device):
            st = fn(*args)
    if st != 0:
        raise DyspecError(st, where)


def _token_rows(t, shape, dtype, device: int, what: str) -> int:
    """Elements between the tokens of t [tokens, heads, d], heads dense."""
    if t.shape != shape or t.dtype is not dtype or t.get_device() != device:
        raise ValueError(f"{what}: {tuple(shape)} of {dtype} on device {device} expected, got {tuple(t.shape)} of {t.dtype} on {t.device}")
    s = t.stride()
    n, heads, d = shape
    if s[2] != 1 or s[1] != d:                 # (of a dimension of one the stride says nothing)
        if (d > 1 and s[2] != 1) or (heads > 1 and s[1] != d):
            raise ValueError(f"{what}: a token's heads must be dense")
    return s[0] if n > 1 else heads * d


def _dense(t, shape, dtype, device: int, what: str) -> int:
    if t.shape != shape or t.dtype is not dtype or t.get_device() != device or not t.is_contiguous():
        raise ValueError(f"{what}: contiguous {tuple(shape)} of {dtype} on device {device} expected, got {tuple(t.shape)} of {t.dtype} on {t.device}")
    return t.data_ptr()


def _chunks(batch: Batch) -> dict:
    """The batch's memo with what the calls below ask for every time: tokens, the C struct by reference."""
    memo = batch._memo()
    if "chunks" not in memo:
        memo["chunks"] = (int(batch.node_offset[-1]), ctypes.byref(batch._c(memo)))
    return memo


def _stream_of(stream, device: int):
    """(raw handle, context in which memory belongs to that stream) of a given stream."""
    if stream.device.index != device:
        raise ValueError("the stream is another device's")
    return int(stream.cuda_stream), _torch.cuda.stream(stream)


_current = contextlib.nullcontext()


def _hand_over(stream, *tensors) -> None:
    """Memory that was given out for other streams is not to be reused while this one reads it."""
    for t in tensors:
        if t is not None:
            t.record_stream(stream)


_attend_scratch: dict = {}


def _attend_workspace(device: int, raw: int, where, nbytes: int, prepared: bool):
    """A paged_attn workspace, its head zero.  Calls of one stream run in order and share one; a prepared call, and a call that a
    graph records, has its own, because whatever runs beside the graph may use the stream's."""
    torch = _torch
    if torch._C._cuda_getDevice() != device:
        with torch.cuda.device(device):
            return _attend_workspace(device, raw, where, nbytes, prepared)
    with where:
        capturing = torch._C._cuda_isCurrentStreamCapturing()
        if not prepared and not capturing:
            buf = _attend_scratch.get((device, raw))
            if buf is not None and buf[1] >= nbytes:
                return buf[0]
        if prepared and capturing:
            raise ValueError("prepare the call before the graph is recorded: its workspace has to be cleared first")
        buf = torch.empty(nbytes, dtype=torch.uint8, device=torch.device("cuda", device))
        buf[:PAGED_COUNTER_BYTES].zero_()                       # (a graph does this at every replay)
        if not prepared and not capturing:
            _attend_scratch[(device, raw)] = (buf, nbytes)
        return buf


def kv_append(k, v, batch: Batch, cache: PagedCache, q=None, rel_pos=None, inv_freq=None, interleaved: bool = False,
              out=None, k_out=None, stream=None):
    """dyspec_kv_append: the new tokens' keys (rotated) and values go into their places in the pages; returns the rotated
    queries (None without q).  k, v [sum N, Hkv, d] and q [sum N, Hq, d] may be slices of one projection's rows.
    rel_pos: int32 positions relative to each sequence's context (a tree's depths), by default 0, 1, ...; inv_freq: fp32 [n],
    the frequencies of the first n pairs of a head (None: nothing is rotated); out: the queries' place (may be q, where that is
    dense); k_out: the rotated keys as dense rows as well."""
    args, out = _append_args(k, v, batch, cache, q, rel_pos, inv_freq, interleaved, out, k_out, stream)
    if args is not None:
        _issue(_lib.dyspec_kv_append, args, cache._device, "dyspec_kv_append")
    return out


def kv_append_call(k, v, batch: Batch, cache: PagedCache, q=None, rel_pos=None, inv_freq=None, interleaved: bool = False,
                   out=None, k_out=None, stream=None) -> PreparedCall:
    """kv_append's call, prepared: nothing is launched until the returned object is called."""
    args, out = _append_args(k, v, batch, cache, q, rel_pos, inv_freq, interleaved, out, k_out, stream)
    if args is None:
        return _Nothing(out)
    keep = (k, v, batch._c(), cache, q, rel_pos, inv_freq, out, k_out)
    return DeviceCall(_lib.dyspec_kv_append, args, keep, "dyspec_kv_append", out, cache._device)


def _append_args(k, v, batch, cache, q, rel_pos, inv_freq, interleaved, out, k_out, stream):
    if _lib is None:
        load_library()
    torch = _torch
    total, ref = _chunks(batch)["chunks"]
    device, dtype, (Hkv, d) = cache._device, cache._torch_dtype, cache._heads
    if cache._layers or cache._rows < batch.n_seq:
        raise ValueError("kv_append takes one layer's cache, with a table row per sequence")
    shape = (total, Hkv, d)
    ks, vs = _token_rows(k, shape, dtype, device, "k"), _token_rows(v, shape, dtype, device, "v")
    raw, where = (torch._C._cuda_getCurrentRawStream(device), _current) if stream is None else _stream_of(stream, device)
    qp = qs = op = Hq = 0
    if q is not None:
        Hq = q.shape[1]
        shape = (total, Hq, d)
        qs, qp = _token_rows(q, shape, dtype, device, "q"), q.data_ptr()
        if out is None:
            with where:
                out = q.new_empty(shape)
            op = out.data_ptr()
        else:
            op = _dense(out, shape, dtype, device, "out")
    elif out is not None:
        raise ValueError("out is the queries' place: q is missing")
    kp = 0 if k_out is None else _dense(k_out, (total, Hkv, d), dtype, device, "k_out")
    rp = 0 if rel_pos is None else _dense(rel_pos, (total,), torch.int32, device, "rel_pos")
    n_freq = fp = 0
    if inv_freq is not None:
        n_freq = inv_freq.numel()
        fp = _dense(inv_freq, (n_freq,), torch.float32, device, "inv_freq")
    if total == 0:
        return None, out
    if stream is not None:
        _hand_over(stream, q, k, v, out, k_out, rel_pos, inv_freq, cache.k, cache.v, cache.page_table)
    return (qp, qs, k.data_ptr(), ks, v.data_ptr(), vs, cache._ref, ref, rp, fp, n_freq, 1 if interleaved else 0, Hq, Hkv, d,
            cache._code, op, kp, raw), out


def kv_keep(cache: PagedCache, batch: Batch, accepted_nodes, n_accepted, stream=None) -> None:
    """dyspec_kv_keep: after verify, the accepted path's rows move up behind the root's, in every layer of the cache.
    `batch` describes the trees as they were appended; accepted_nodes and n_accepted are verify's."""
    if _lib is None:
        load_library()
    torch = _torch
    total, ref = _chunks(batch)["chunks"]
    device, (Hkv, d), n_seq = cache._device, cache._heads, batch.n_seq
    if cache._rows < n_seq:
        raise ValueError("a table row per sequence is needed")
    ap = _dense(accepted_nodes, (total,), torch.int32, device, "accepted_nodes")
    np_ = _dense(n_accepted, (n_seq,), torch.int32, device, "n_accepted")
    if total == 0:
        return
    if stream is None:
        raw = torch._C._cuda_getCurrentRawStream(device)
    else:
        raw, _ = _stream_of(stream, device)
        _hand_over(stream, accepted_nodes, n_accepted, cache.k, cache.v, cache.page_table)
    _issue(_lib.dyspec_kv_keep, (cache._ref, cache._layers or 1, cache._layer_stride, ref, ap, np_, Hkv, d, cache._code, raw), device, "dyspec_kv_keep")


def paged_attn(q, batch: Batch, cache: PagedCache, softmax_scale: float, anc_mask=None, out=None, stream=None, cap: Optional[float] = None,
               window: Optional[int] = None, rel_pos=None):
    """dyspec_paged_attn, with cap or window dyspec_paged_attn_scored: the new tokens (appended before) attend to the pages: to their
    context and, causally or by an ancestor mask [sum N, max(1, ceil(max N / 64))], to each other.  q/out [sum N, Hq, d].
    cap: scores s count as cap * tanh(s / cap); window: of keys less than that many positions back; rel_pos: int32 [sum N] positions of
    the new tokens relative to each sequence's context (a tree's depths, as for kv_append; only a window reads them), by default 0, 1, ..."""
    args, out, _ = _attn_args(q, batch, cache, softmax_scale, anc_mask, out, stream, False, cap, window, rel_pos)
    if args is not None:
        if cap is None and window is None:
            _issue(_lib.dyspec_paged_attn, args, cache._device, "dyspec_paged_attn")
        else:
            _issue(_lib.dyspec_paged_attn_scored, args, cache._device, "dyspec_paged_attn_scored")
    return out


def paged_attn_call(q, batch: Batch, cache: PagedCache, softmax_scale: float, anc_mask=None, out=None, stream=None, cap: Optional[float] = None,
                    window: Optional[int] = None, rel_pos=None) -> PreparedCall:
    """paged_attn's call, prepared: nothing is launched until the returned object is called.  It has a workspace of its own."""
    where = "dyspec_paged_attn" if cap is None and window is None else "dyspec_paged_attn_scored"
    args, out, ws = _attn_args(q, batch, cache, softmax_scale, anc_mask, out, stream, True, cap, window, rel_pos)
    if args is None:
        return _Nothing(out)
    return DeviceCall(getattr(_lib, where), args, (q, batch._c(), cache, anc_mask, out, ws, rel_pos), where, out, cache._device)


def _scores(cap, window, rel_pos, total: int, device: int):
    """The C struct for capped scores and windows; None where there are neither.  (rel_pos is looked at all the same: a layer without a
    window takes the call of one that has it, as it is.)"""
    if window is not None and not window >= 1:
        raise ValueError("window: at least 1, or None")
    rp = 0 if rel_pos is None else _dense(rel_pos, (total,), _torch.int32, device, "rel_pos")
    if cap is None and window is None:
        return None
    x = _Scores(cap or 0.0, min(window or 0, (1 << 31) - 1), rp)
    if cap is not None and not x.cap > 0:                          # (as the call has it: what rounds to zero would be none)
        raise ValueError("cap: a positive number of 32 bits, or None")
    return x


def _attn_args(q, batch, cache, softmax_scale, anc_mask, out, stream, prepared, cap=None, window=None, rel_pos=None):
    if _lib is None:
        load_library()
    torch = _torch
    memo = _chunks(batch)
    total, ref = memo["chunks"]
    device, dtype, (Hkv, d), code = cache._device, cache._torch_dtype, cache._heads, cache._code
    if cache._layers or cache._rows < batch.n_seq:
        raise ValueError("paged_attn takes one layer's cache, with a table row per sequence")
    Hq = q.shape[1]
    shape = (total, Hq, d)
    qp = _dense(q, shape, dtype, device, "q")
    mp = 0
    if anc_mask is not None:
        words = memo.get("chunk_words")
        if words is None:
            words = memo["chunk_words"] = max(1, -(-int(np.diff(batch.node_offset).max()) // 64))
        mp = _dense(anc_mask, (total, words), torch.int64, device, "anc_mask")
    raw, where = (torch._C._cuda_getCurrentRawStream(device), _current) if stream is None else _stream_of(stream, device)
    scores = None if cap is None and window is None and rel_pos is None else _scores(cap, window, rel_pos, total, device)
    if out is None:
        with where:
            out = torch.empty_like(q)
        op = out.data_ptr()
    else:
        op = _dense(out, shape, dtype, device, "out")
    if total == 0:
        return None, out, None
    key = ("ws_paged", Hq, Hkv, d, code) if scores is None else ("ws_paged", Hq, Hkv, d, code, scores.cap, scores.window, rel_pos is None)
    nbytes = memo.get(key)
    if nbytes is None:
        nbytes = memo[key] = int(_lib.dyspec_paged_attn_workspace_bytes(ref, Hq, Hkv, d, code) if scores is None else
                                 _lib.dyspec_paged_attn_scored_workspace_bytes(ref, Hq, Hkv, d, code, scores))
    ws, wp = None, 0
    if nbytes:
        ws = _attend_workspace(device, raw, where, nbytes, prepared)
        wp = ws.data_ptr()
    if stream is not None:
        _hand_over(stream, q, out, anc_mask, rel_pos, cache.k, cache.v, cache.page_table)
    if scores is None:
        return (qp, cache._ref, ref, mp, Hq, Hkv, d, code, softmax_scale, op, wp, nbytes, raw), out, ws
    return (qp, cache._ref, ref, mp, Hq, Hkv, d, code, softmax_scale, scores, op, wp, nbytes, raw), out, ws


def prompt_attn(q, k, v, batch: Batch, softmax_scale: float, out=None, stream=None, cap: Optional[float] = None, window: Optional[int] = None, rel_pos=None):
    """dyspec_prompt_attn, with cap or window dyspec_prompt_attn_scored: packed prompts attend to themselves, causally.  q [sum N, Hq, d],
    k, v [sum N, Hkv, d], which may be slices of one projection's rows; the batch's n_nodes are the prompts' lengths, its prefix_len
    zeros.  cap, window, rel_pos as for paged_attn."""
    args, out, device = _prompt_args(q, k, v, batch, softmax_scale, out, stream, cap, window, rel_pos)
    if args is not None:
        if cap is None and window is None:
            _issue(_lib.dyspec_prompt_attn, args, device, "dyspec_prompt_attn")
        else:
            _issue(_lib.dyspec_prompt_attn_scored, args, device, "dyspec_prompt_attn_scored")
    return out


def prompt_attn_call(q, k, v, batch: Batch, softmax_scale: float, out=None, stream=None, cap: Optional[float] = None, window: Optional[int] = None,
                     rel_pos=None) -> PreparedCall:
    """prompt_attn's call, prepared: nothing is launched until the returned object is called."""
    where = "dyspec_prompt_attn" if cap is None and window is None else "dyspec_prompt_attn_scored"
    args, out, device = _prompt_args(q, k, v, batch, softmax_scale, out, stream, cap, window, rel_pos)
    if args is None:
        return _Nothing(out)
    return DeviceCall(getattr(_lib, where), args, (q, k, v, batch._c(), out, rel_pos), where, out, device)


def _prompt_args(q, k, v, batch, softmax_scale, out, stream, cap=None, window=None, rel_pos=None):
    if _lib is None:
        load_library()
    total, ref = _chunks(batch)["chunks"]
    device, dtype = q.get_device(), q.dtype
    if device < 0:
        raise ValueError("device tensor required")
    code = _code(dtype)
    _, Hq, d = q.shape
    Hkv = k.shape[1]
    shape, kv_shape = (total, Hq, d), (total, Hkv, d)
    qs = _token_rows(q, shape, dtype, device, "q")
    ks, vs = _token_rows(k, kv_shape, dtype, device, "k"), _token_rows(v, kv_shape, dtype, device, "v")
    raw, where = (_torch._C._cuda_getCurrentRawStream(device), _current) if stream is None else _stream_of(stream, device)
    if out is None:
        with where:
            out = q.new_empty(shape)
        op = out.data_ptr()
    else:
        op = _dense(out, shape, dtype, device, "out")
    scores = None if cap is None and window is None and rel_pos is None else _scores(cap, window, rel_pos, total, device)
    if total == 0:
        return None, out, device
    if stream is not None:
        _hand_over(stream, q, k, v, out, rel_pos)
    if scores is None:
        return (q.data_ptr(), qs, k.data_ptr(), ks, v.data_ptr(), vs, ref, Hq, Hkv, d, code, softmax_scale, op, raw), out, device
    return (q.data_ptr(), qs, k.data_ptr(), ks, v.data_ptr(), vs, ref, Hq, Hkv, d, code, softmax_scale, scores, op, raw), out, device


# ---------------------------------------------------------------------------------------- pages by the requests' lengths

@dataclass(frozen=True)
class PagePool:
    """The free pages of a pool, as a ring on the device (see dyspec_page_pool in include/dyspec.h).

    ring   int32 [n_pages]: page numbers, the free ones from state[0] on, round the end
    state  int32 [4]: first free place of the ring, number of free pages, 0, 0"""
    ring: "torch.Tensor"
    state: "torch.Tensor"
    page_size: int

    def __post_init__(self):
        ring, state = self.ring, self.state
        i32 = _dtype("int32")
        if ring.dim() != 1 or ring.numel() < 1 or ring.dtype is not i32 or not ring.is_cuda or not ring.is_contiguous():
            raise ValueError("ring must be a contiguous int32 device tensor [n_pages]")
        if state.shape != (4,) or state.dtype is not i32 or state.device != ring.device or not state.is_contiguous():
            raise ValueError("state must be a contiguous int32 tensor [4] on the ring's device")
        c = _PagePool(ring.data_ptr(), state.data_ptr(), int(ring.numel()), int(self.page_size))
        for name, value in dict(_c=c, _ref=ctypes.byref(c), _device=ring.get_device()).items():
            object.__setattr__(self, name, value)

    @staticmethod
    def full(n_pages: int, page_size: int, device) -> "PagePool":
        """A pool of which every page is free."""
        import torch
        ring = torch.arange(n_pages, dtype=torch.int32, device=device)
        return PagePool(ring, torch.tensor([0, n_pages, 0, 0], dtype=torch.int32, device=ring.device), page_size)


def page_plan(pool: PagePool, page_table, held, wanted, slots=None, granted=None, stream=None, slots_from=None):
    """dyspec_page_plan: every sequence gets pages for wanted[s] tokens in place of held[s], from the pool or back to it; returns
    granted [n_seq], the tokens that it now has pages for (held[s] where the pool was short, -1 for lengths that cannot be).
    page_table: int32 [n_seq or more, max_pages], a PagedCache's; held, wanted: int32 [n_seq]; slots: int64 [any], where the new
    tokens' rows of the pool are noted, packed by sequences: of tokens slots_from[s] (int32 [n_seq]; None: held[s]) to wanted[s] - 1."""
    args, granted = _plan_args(pool, page_table, held, wanted, slots, granted, stream, slots_from)
    _issue(_lib.dyspec_page_plan, args, pool._device, "dyspec_page_plan")
    return granted


def page_plan_call(pool: PagePool, page_table, held, wanted, slots=None, granted=None, stream=None, slots_from=None) -> PreparedCall:
    """page_plan's call, prepared: nothing is launched until the returned object is called."""
    args, granted = _plan_args(pool, page_table, held, wanted, slots, granted, stream, slots_from)
    return DeviceCall(_lib.dyspec_page_plan, args, (pool, page_table, held, wanted, slots, granted, slots_from), "dyspec_page_plan", granted, pool._device)


def _plan_args(pool, page_table, held, wanted, slots, granted, stream, slots_from):
    if _lib is None:
        load_library()
    torch = _torch
    device, n_seq, rows = pool._device, held.numel(), page_table.shape
    if len(rows) != 2 or rows[0] < n_seq or page_table.dtype is not torch.int32 or page_table.get_device() != device or (rows[1] > 1 and page_table.stride(1) != 1):
        raise ValueError("page_table: int32 [n_seq or more, max_pages] on the pool's device expected")
    hp, wp = _dense(held, (n_seq,), torch.int32, device, "held"), _dense(wanted, (n_seq,), torch.int32, device, "wanted")
    fp = 0 if slots_from is None else _dense(slots_from, (n_seq,), torch.int32, device, "slots_from")
    sp = n_slots = 0
    if slots is not None:
        n_slots = slots.numel()
        sp = _dense(slots, (n_slots,), torch.int64, device, "slots")
    raw, where = (torch._C._cuda_getCurrentRawStream(device), _current) if stream is None else _stream_of(stream, device)
    if granted is None:
        with where:
            granted = torch.empty_like(held)
        gp = granted.data_ptr()
    else:
        gp = _dense(granted, (n_seq,), torch.int32, device, "granted")
    if stream is not None:
        _hand_over(stream, pool.ring, pool.state, page_table, held, wanted, slots, granted, slots_from)
    return (pool._ref, page_table.data_ptr(), rows[1], page_table.stride(0) if rows[0] > 1 else rows[1], hp, wp, n_seq, gp, sp, n_slots, fp, raw), granted


# ---------------------------------------------------------------------------------------- filtered logits and drawn tokens

@dataclass
class Sampled:
    token: "torch.Tensor"          # int32 [rows]; -1: the row has no distribution
    prob: "torch.Tensor"           # fp32 [rows]: its probability among the tokens that are kept
    n_kept: "torch.Tensor"         # int32 [rows]

    @staticmethod
    def empty(rows: int, device) -> "Sampled":
        import torch
        i = lambda: torch.empty(rows, dtype=torch.int32, device=device)
        return Sampled(i(), torch.empty(rows, dtype=torch.float32, device=device), i())


def sample(logits, batch: Batch, uniform, temperature, top_k=None, top_p=None, min_p=None, out: Optional[Sampled] = None, stream=None) -> Sampled:
    """dyspec_sample: a token for every row of logits [rows, vocab] (a batch's n_nodes are its sequences' rows) by the given random
    numbers uniform [rows] fp32 in [0, 1), after temperature, top-k, top-p and min-p: a number for all sequences, or one each; None:
    no such filter.  These settings are read on the host when the call is made or prepared (a recorded graph keeps its own)."""
    args, out, device, _ = _sample_args(logits, batch, uniform, temperature, top_k, top_p, min_p, out, stream)
    if args is not None:
        _issue(_lib.dyspec_sample, args, device, "dyspec_sample")
    return out


def sample_call(logits, batch: Batch, uniform, temperature, top_k=None, top_p=None, min_p=None, out: Optional[Sampled] = None, stream=None) -> PreparedCall:
    """sample's call, prepared: nothing is launched until the returned object is called."""
    args, out, device, held = _sample_args(logits, batch, uniform, temperature, top_k, top_p, min_p, out, stream)
    if args is None:
        return _Nothing(out)
    return DeviceCall(_lib.dyspec_sample, args, (logits, uniform, batch._c(), held, out), "dyspec_sample", out, device)


def filter_logits(logits, batch: Batch, temperature, top_k=None, top_p=None, min_p=None, out=None, stream=None):
    """dyspec_filter_logits: logits [rows, vocab] with -inf in place of what top-k, top-p and min-p take out (settings as for
    sample); build_tree and verify on such tables, at the same temperatures, draw from the filtered distributions.  out: may be
    logits."""
    args, out, device, _ = _filter_args(logits, batch, temperature, top_k, top_p, min_p, out, stream)
    if args is not None:
        _issue(_lib.dyspec_filter_logits, args, device, "dyspec_filter_logits")
    return out


def filter_logits_call(logits, batch: Batch, temperature, top_k=None, top_p=None, min_p=None, out=None, stream=None) -> PreparedCall:
    """filter_logits' call, prepared: nothing is launched until the returned object is called."""
    args, out, device, held = _filter_args(logits, batch, temperature, top_k, top_p, min_p, out, stream)
    if args is None:
        return _Nothing(out)
    return DeviceCall(_lib.dyspec_filter_logits, args, (logits, batch._c(), held, out), "dyspec_filter_logits", out, device)


def _per_sequence(x, code: str, n_seq: int, what: str):
    """One number a sequence as C has them ('f': fp32, 'i': int32), None for None."""
    if x is None:
        return None
    if isinstance(x, (int, float)):
        x = (x,) * n_seq
    elif not isinstance(x, (list, tuple)):
        try:
            x = np.asarray(x).tolist()
        except (TypeError, RuntimeError):                          # (a device's tensor, one with a gradient)
            raise ValueError(f"{what}: numbers on the host expected, got {type(x).__name__}") from None
        if not isinstance(x, list):
            x = (x,) * n_seq
    if len(x) != n_seq:
        raise ValueError(f"{what}: a number, or one for each of the {n_seq} sequences expected")
    try:
        return struct.pack(f"{n_seq}{code}", *x)                   # (64 of them 1 us, as a ctypes array 4.4)
    except (struct.error, OverflowError) as e:
        raise ValueError(f"{what}: 32-bit numbers expected ({e})") from None


def _settings(batch, temperature, top_k, top_p, min_p):
    n = batch.n_seq
    return (_per_sequence(temperature, "f", n, "temperature"), _per_sequence(top_k, "i", n, "top_k"),
            _per_sequence(top_p, "f", n, "top_p"), _per_sequence(min_p, "f", n, "min_p"))


def _logit_rows(t, total: int, what: str) -> int:
    """Elements between the rows of t [total, vocab], each dense."""
    if t.dim() != 2 or t.shape[0] != total or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError(f"{what}: a dense row for each of the batch's {total} expected, got {tuple(t.shape)}")
    return t.stride(0) if total > 1 else t.shape[1]


def _sample_args(logits, batch, uniform, temperature, top_k, top_p, min_p, out, stream):
    if _lib is None:
        load_library()
    torch = _torch
    total, ref = _chunks(batch)["chunks"]
    device = logits.get_device()
    if device < 0:
        raise ValueError("device tensor required")
    code, stride = _code(logits.dtype), _logit_rows(logits, total, "logits")
    up = _dense(uniform, (total,), torch.float32, device, "uniform")
    held = _settings(batch, temperature, top_k, top_p, min_p)
    raw, where = (torch._C._cuda_getCurrentRawStream(device), _current) if stream is None else _stream_of(stream, device)
    if out is None:
        with where:
            out = Sampled(uniform.new_empty(total, dtype=torch.int32), uniform.new_empty(total), uniform.new_empty(total, dtype=torch.int32))
        tp, pp, np_ = out.token.data_ptr(), out.prob.data_ptr(), out.n_kept.data_ptr()
    else:
        tp, pp = _dense(out.token, (total,), torch.int32, device, "token"), _dense(out.prob, (total,), torch.float32, device, "prob")
        np_ = _dense(out.n_kept, (total,), torch.int32, device, "n_kept")
    if total == 0:
        return None, out, device, held
    if stream is not None:
        _hand_over(stream, logits, uniform, out.token, out.prob, out.n_kept)
    return (logits.data_ptr(), code, logits.shape[1], stride, ref, *held, up, tp, pp, np_, raw), out, device, held


def _filter_args(logits, batch, temperature, top_k, top_p, min_p, out, stream):
    if _lib is None:
        load_library()
    torch = _torch
    total, ref = _chunks(batch)["chunks"]
    device = logits.get_device()
    if device < 0:
        raise ValueError("device tensor required")
    code, stride = _code(logits.dtype), _logit_rows(logits, total, "logits")
    held = _settings(batch, temperature, top_k, top_p, min_p)
    raw, where = (torch._C._cuda_getCurrentRawStream(device), _current) if stream is None else _stream_of(stream, device)
    if out is None:
        with where:
            out = logits.new_empty(logits.shape)
        out_stride = logits.shape[1]
    else:
        if out.shape != logits.shape or out.dtype is not logits.dtype or out.get_device() != device:
            raise ValueError("out: a table like logits expected")
        out_stride = _logit_rows(out, total, "out")
    if total == 0:
        return None, out, device, held
    if stream is not None:
        _hand_over(stream, logits, out)
    return (logits.data_ptr(), code, logits.shape[1], stride, ref, *held, out.data_ptr(), out_stride, raw), out, device, held


def probe_mfma_bf16(iterations: int, sink, stream=None, random_operands: bool = False) -> float:
    """dyspec_probe_mfma_bf16: launches the MFMA-only loop, returns the flops of the launch."""
    flops = ctypes.c_double(0.0)
    _check(load_library().dyspec_probe_mfma_bf16(int(iterations), int(bool(random_operands)), ctypes.byref(flops),
                                                 _ptr(sink, "float32"), _stream(stream)), "dyspec_probe_mfma_bf16")
    return float(flops.value)


def probe_clock(iterations: int, counters, stream=None) -> int:
    """dyspec_probe_clock: launches the sleeping wave; counters (int64[2], device) receives shader
    cycles and wall clock ticks once it ends.  Returns the wall clock rate in kHz."""
    khz = ctypes.c_int32(0)
    _check(load_library().dyspec_probe_clock(int(iterations), _ptr(counters, "int64"), ctypes.byref(khz), _stream(stream)),
           "dyspec_probe_clock")
    return int(khz.value)


def probe_hbm_read(src, sink, stream=None) -> int:
    """dyspec_probe_hbm_read: launches one streaming read of src, returns the bytes read."""
    nbytes = (src.numel() * src.element_size()) // 16 * 16
    _check(load_library().dyspec_probe_hbm_read(_ptr(src), ctypes.c_size_t(nbytes), _ptr(sink, "float32"),
                                                _stream(stream)), "dyspec_probe_hbm_read")
    return nbytes
