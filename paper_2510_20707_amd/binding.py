"""ctypes binding of libmixkv (see include/mixkv.h).  Argument marshalling only.

Every function here has the name of the C entry point it calls and does nothing
but build the C structs from torch tensors (device memory and the current HIP
stream come from torch) and check the returned status.  There is no fallback:
if the shared library has not been built, `lib()` raises.
"""
from __future__ import annotations

import ctypes as C
import operator
import os
from array import array
from dataclasses import dataclass, is_dataclass
from typing import List, Optional, Sequence

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmixkv.so")

MIXKV_OK, MIXKV_ERR_INVALID_ARG, MIXKV_ERR_UNSUPPORTED, MIXKV_ERR_WORKSPACE_TOO_SMALL, MIXKV_ERR_HIP = range(5)
DTYPE = {"f32": 0, "bf16": 1}
POOL = {"none": 0, "avg": 1, "max": 2}
BUDGET_MODE = {"fixed": 0, "adaptive": 1, "per_head": 2}
INTRINSIC = {"none": 0, "vnorm": 1, "knorm": 2}
MIX = {"head_adaptive": 0, "sum": 1, "div_only": 2, "imp_only": 3, "given_r": 4}
TORCH_DTYPE = {0: torch.float32, 1: torch.bfloat16}
PAGE_FORMAT = {"rows": 0, "4bit": 1}
N_STAGES = 5


class MixkvParams(C.Structure):
    _fields_ = [
        ("dtype", C.c_int), ("batch", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32),
        ("head_dim", C.c_int32), ("seq_len", C.c_int32), ("window", C.c_int32), ("budget", C.c_int32),
        ("pool", C.c_int), ("pool_kernel", C.c_int32), ("causal_window", C.c_int32),
        ("softmax_scale", C.c_float), ("eps", C.c_float), ("intrinsic", C.c_int), ("mix", C.c_int),
        ("budget_mode", C.c_int), ("budget_floor", C.c_int32), ("head_budgets", C.c_void_p),
    ]


class MixkvLayerIn(C.Structure):
    _fields_ = [("K", C.c_void_p), ("V", C.c_void_p), ("kv_stride_b", C.c_int64), ("kv_stride_h", C.c_int64),
                ("kv_stride_n", C.c_int64), ("Qwin", C.c_void_p), ("r_given", C.c_void_p),
                ("window_lse", C.c_void_p)]


class MixkvLayerOut(C.Structure):
    _fields_ = [("scores", C.c_void_p), ("redundancy", C.c_void_p), ("indices", C.c_void_p), ("counts", C.c_void_p),
                ("offsets", C.c_void_p), ("K_out", C.c_void_p), ("V_out", C.c_void_p)]


class MixkvRowsIn(C.Structure):
    _fields_ = [("X", C.c_void_p), ("stride_b", C.c_int64), ("stride_h", C.c_int64), ("stride_n", C.c_int64)]


class MixkvSimilarityOut(C.Structure):
    _fields_ = [("redundancy", C.c_void_p), ("block_map", C.c_void_p)]


class MixkvDecodeLayer(C.Structure):
    _fields_ = [("K_cache", C.c_void_p), ("V_cache", C.c_void_p), ("counts", C.c_void_p), ("offsets", C.c_void_p),
                ("K_tail", C.c_void_p), ("V_tail", C.c_void_p), ("Q", C.c_void_p), ("out", C.c_void_p)]


class MixkvAppendLayer(C.Structure):
    _fields_ = [("K_new", C.c_void_p), ("V_new", C.c_void_p), ("K_tail", C.c_void_p), ("V_tail", C.c_void_p)]


class MixkvPagedParams(C.Structure):
    _fields_ = [("dtype", C.c_int), ("format", C.c_int), ("batch", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("page_rows", C.c_int32), ("max_pages", C.c_int32), ("n_pages", C.c_int32),
                ("softmax_scale", C.c_float)]


class MixkvPagedCache(C.Structure):
    _fields_ = [("K_pages", C.c_void_p), ("V_pages", C.c_void_p), ("K_bounds", C.c_void_p), ("page_table", C.c_void_p),
                ("lengths", C.c_void_p)]


class MixkvPagedRows(C.Structure):
    _fields_ = [("K", C.c_void_p), ("V", C.c_void_p), ("stride_n", C.c_int64), ("stride_h", C.c_int64), ("row_start", C.c_void_p),
                ("row_count", C.c_void_p), ("Q", C.c_void_p), ("q_stride_n", C.c_int64), ("q_stride_h", C.c_int64), ("Q_out", C.c_void_p)]


class MixkvRope(C.Structure):
    _fields_ = [("cos", C.c_void_p), ("sin", C.c_void_p), ("n_positions", C.c_int32), ("positions", C.c_void_p), ("n_axes", C.c_int32),
                ("sections", C.c_int32 * 3)]


class MixkvPagedSelectLayer(C.Structure):
    _fields_ = [("Q", C.c_void_p), ("selected", C.c_void_p), ("n_selected", C.c_void_p)]


class MixkvPagedAttentionLayer(C.Structure):
    _fields_ = [("Q", C.c_void_p), ("out", C.c_void_p), ("selected", C.c_void_p), ("n_selected", C.c_void_p)]


class MixkvPagedQueries(C.Structure):
    _fields_ = [("Q", C.c_void_p), ("q_stride_n", C.c_int64), ("q_stride_h", C.c_int64), ("row_start", C.c_void_p), ("row_count", C.c_void_p),
                ("out", C.c_void_p), ("lse", C.c_void_p)]


class MixkvPagedEvictLayer(C.Structure):
    _fields_ = [("weights", C.c_void_p), ("weights_into", C.c_void_p), ("keep", C.c_void_p), ("kept", C.c_void_p), ("n_kept", C.c_void_p)]


class MixkvError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status})")


_lib = None


def lib() -> C.CDLL:
    """Load libmixkv.so (built by `python -m paper_2510_20707_amd.build`)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2510_20707_amd.build`")
        L = C.CDLL(LIB_PATH)
        pp, pin, pout = C.POINTER(MixkvParams), C.POINTER(MixkvLayerIn), C.POINTER(MixkvLayerOut)
        L.mixkv_workspace_size.argtypes = [pp, C.c_int32, C.POINTER(C.c_size_t)]
        L.mixkv_workspace_size.restype = C.c_int
        L.mixkv_score.argtypes = [pp, pin, pout, C.c_int32, C.c_void_p, C.c_size_t, C.c_void_p]
        L.mixkv_score.restype = C.c_int
        L.mixkv_select.argtypes = [pp, pout, C.c_int32, C.c_void_p, C.c_size_t, C.c_void_p]
        L.mixkv_select.restype = C.c_int
        L.mixkv_compress.argtypes = [pp, pin, pout, C.c_int32, C.c_void_p, C.c_size_t, C.c_void_p]
        L.mixkv_compress.restype = C.c_int
        L.mixkv_compress_static.argtypes = [pp, pin, pout, C.c_int32, C.c_void_p]
        L.mixkv_compress_static.restype = C.c_int
        L.mixkv_compress_profiled.argtypes = [pp, pin, pout, C.c_int32, C.c_void_p, C.c_size_t, C.c_void_p,
                                              C.POINTER(C.c_float)]
        L.mixkv_compress_profiled.restype = C.c_int
        L.mixkv_similarity_workspace_size.argtypes = [pp, C.c_int32, C.c_int32, C.POINTER(C.c_size_t)]
        L.mixkv_similarity_workspace_size.restype = C.c_int
        L.mixkv_similarity.argtypes = [pp, C.POINTER(MixkvRowsIn), C.POINTER(MixkvSimilarityOut), C.c_int32, C.c_int32,
                                       C.c_void_p, C.c_size_t, C.c_void_p]
        L.mixkv_similarity.restype = C.c_int
        L.mixkv_decode_attention.argtypes = [pp, C.POINTER(MixkvDecodeLayer), C.c_int32, C.c_int32, C.c_int32, C.c_void_p,
                                             C.c_size_t, C.c_void_p]
        L.mixkv_decode_attention.restype = C.c_int
        L.mixkv_append.argtypes = [pp, C.POINTER(MixkvAppendLayer), C.c_int32, C.c_int32, C.c_int32, C.c_void_p]
        L.mixkv_append.restype = C.c_int
        L.mixkv_decode_workspace_size.argtypes = [pp, C.c_int32, C.c_int32, C.POINTER(C.c_size_t)]
        L.mixkv_decode_workspace_size.restype = C.c_int
        pg, pc, pr = C.POINTER(MixkvPagedParams), C.POINTER(MixkvPagedCache), C.POINTER(MixkvPagedRows)
        L.mixkv_page_bytes.argtypes = [pg, C.POINTER(C.c_size_t)]
        L.mixkv_page_bytes.restype = C.c_int
        L.mixkv_paged_append.argtypes = [pg, pc, pr, C.c_int32, C.POINTER(MixkvRope), C.c_int32, C.c_int32, C.c_void_p]
        L.mixkv_paged_append.restype = C.c_int
        L.mixkv_paged_read.argtypes = [pg, pc, pr, C.c_int32, C.c_int32, C.c_int32, C.c_void_p]
        L.mixkv_paged_read.restype = C.c_int
        L.mixkv_paged_select_workspace_size.argtypes = [pg, C.c_int32, C.POINTER(C.c_size_t)]
        L.mixkv_paged_select_workspace_size.restype = C.c_int
        L.mixkv_paged_select.argtypes = [pg, pc, C.POINTER(MixkvPagedSelectLayer), C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_void_p,
                                         C.c_size_t, C.c_void_p]
        L.mixkv_paged_select.restype = C.c_int
        L.mixkv_paged_attention_workspace_size.argtypes = [pg, C.c_int32, C.c_int32, C.POINTER(C.c_size_t)]
        L.mixkv_paged_attention_workspace_size.restype = C.c_int
        L.mixkv_paged_attention.argtypes = [pg, pc, C.POINTER(MixkvPagedAttentionLayer), C.c_int32, C.c_int32, C.c_int32, C.c_void_p,
                                            C.c_size_t, C.c_void_p]
        L.mixkv_paged_attention.restype = C.c_int
        pq, pe, ints = C.POINTER(MixkvPagedQueries), C.POINTER(MixkvPagedEvictLayer), [C.c_int32] * 6
        for name in ("mixkv_paged_window_attention_workspace_size", "mixkv_paged_weights_workspace_size"):
            getattr(L, name).argtypes = [pg, *ints, C.POINTER(C.c_size_t)]
            getattr(L, name).restype = C.c_int
        L.mixkv_paged_window_attention.argtypes = [pg, pc, pq, *ints, C.c_void_p, C.c_size_t, C.c_void_p]
        L.mixkv_paged_window_attention.restype = C.c_int
        L.mixkv_paged_weights.argtypes = [pg, pc, pq, C.POINTER(C.c_void_p), *ints, C.c_void_p, C.c_size_t, C.c_void_p]
        L.mixkv_paged_weights.restype = C.c_int
        L.mixkv_paged_evict_workspace_size.argtypes = [pg, C.c_int32, C.c_int32, C.POINTER(C.c_size_t)]
        L.mixkv_paged_evict_workspace_size.restype = C.c_int
        L.mixkv_paged_evict.argtypes = [pg, pc, pc, pe, *[C.c_int32] * 5, C.c_void_p, C.c_size_t, C.c_void_p]
        L.mixkv_paged_evict.restype = C.c_int
        L.mixkv_stage_name.argtypes = [C.c_int32]
        L.mixkv_stage_name.restype = C.c_char_p
        L.mixkv_status_string.argtypes = [C.c_int]
        L.mixkv_status_string.restype = C.c_char_p
        L.mixkv_version.argtypes = []
        L.mixkv_version.restype = C.c_int32
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().mixkv_status_string(status).decode()


def make_params(dtype: str, batch: int, n_q_heads: int, n_kv_heads: int, head_dim: int, seq_len: int, window: int,
                budget: int, pool: str = "max", pool_kernel: int = 7, causal_window: bool = True,
                softmax_scale: float = 1.0, eps: float = 1e-6, intrinsic: str = "vnorm",
                budget_mode: str = "fixed", budget_floor: int = 0, mix: str = "head_adaptive",
                head_budgets=None) -> MixkvParams:
    """`head_budgets`: host int32 array [n_layers, n_kv_heads] for budget mode "per_head"."""
    p = MixkvParams(DTYPE[dtype], batch, n_q_heads, n_kv_heads, head_dim, seq_len, window, budget, POOL[pool],
                    pool_kernel, int(causal_window), softmax_scale, eps, INTRINSIC[intrinsic], MIX[mix],
                    BUDGET_MODE[budget_mode], budget_floor, None)
    if head_budgets is not None:
        hb = np.ascontiguousarray(head_budgets, dtype=np.int32)
        assert hb.ndim == 2 and hb.shape[1] == n_kv_heads
        p._head_budgets_keep = hb                   # the struct only holds the address
        p.head_budgets = hb.ctypes.data
    return p


@dataclass
class LayerOut:
    """Device tensors receiving one layer's outputs; members may be None where the C API allows NULL."""
    scores: Optional[torch.Tensor] = None        # [batch, Hkv, N] f32
    redundancy: Optional[torch.Tensor] = None    # [batch, Hkv] f32
    indices: Optional[torch.Tensor] = None       # [batch, Hkv, B] i32 (adaptive: packed per batch item)
    counts: Optional[torch.Tensor] = None        # [batch, Hkv] i32
    offsets: Optional[torch.Tensor] = None       # [batch, Hkv + 1] i32
    K_out: Optional[torch.Tensor] = None         # [batch, Hkv, B, D]
    V_out: Optional[torch.Tensor] = None


def alloc_layer_out(p: MixkvParams, device, scores=True, redundancy=True, select=True, gather=True) -> LayerOut:
    """Allocate one layer's outputs with torch (plumbing for tests and the benchmark)."""
    o = LayerOut()
    bt, h, n, b, d = p.batch, p.n_kv_heads, p.seq_len, p.budget, p.head_dim
    if scores:
        o.scores = torch.empty((bt, h, n), dtype=torch.float32, device=device)
    if redundancy:
        o.redundancy = torch.empty((bt, h), dtype=torch.float32, device=device)
    if select:
        o.indices = torch.empty((bt, h, b), dtype=torch.int32, device=device)
        o.counts = torch.empty((bt, h), dtype=torch.int32, device=device)
        o.offsets = torch.empty((bt, h + 1), dtype=torch.int32, device=device)
    if gather:
        o.K_out = torch.empty((bt, h, b, d), dtype=TORCH_DTYPE[p.dtype], device=device)
        o.V_out = torch.empty((bt, h, b, d), dtype=TORCH_DTYPE[p.dtype], device=device)
    return o


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else C.c_void_p(t.data_ptr())


def _address(t: Optional[torch.Tensor]) -> int:
    return 0 if t is None else t.data_ptr()


def _structs(struct, n: int, words):
    """An array of n `struct`, whose fields are all pointers or int64, over its words (zeros for those not given): the words'
    own buffer, where building it field by field takes as long as a short call's kernels."""
    size = C.sizeof(struct) // 8 * n
    return (struct * n).from_buffer(array("q", words if len(words) == size else list(words) + [0] * (size - len(words))))


def _in_array(Ks, Vs, Qs, r_given=None, window_lse=None):
    """r_given: per layer a contiguous f32 [batch, Hkv] device tensor (mix "given_r"), or None;
    window_lse: per layer a contiguous f32 [batch, Hq, W] device tensor, or None."""
    words = []
    for i, (K, V, Q) in enumerate(zip(Ks, Vs, Qs)):
        strides = K.stride()
        assert K.dim() == 4 and strides[3] == 1 and V.shape == K.shape and V.stride() == strides
        assert Q is None or Q.is_contiguous()
        rg = None if r_given is None else r_given[i]
        assert rg is None or (rg.is_contiguous() and rg.dtype == torch.float32 and rg.shape == K.shape[:2])
        lse = None if window_lse is None else window_lse[i]
        assert lse is None or (lse.is_contiguous() and lse.dtype == torch.float32 and lse.shape == Q.shape[:3])
        words += (K.data_ptr(), V.data_ptr(), strides[0], strides[1], strides[2], _address(Q), _address(rg), _address(lse))
    return _structs(MixkvLayerIn, len(Ks), words)


_out_members = operator.attrgetter(*(name for name, _ in MixkvLayerOut._fields_))


def _out_array(outs: Sequence[LayerOut]):
    return _structs(MixkvLayerOut, len(outs), [0 if t is None else t.data_ptr() for o in outs for t in _out_members(o)])


def _stream(stream) -> C.c_void_p:
    if stream is None:
        # the current stream's handle without the stream object around it (2.9 -> 0.4 us, a third of a decoding step's host time)
        return C.c_void_p(torch._C._cuda_getCurrentRawStream(torch.cuda.current_device()))
    return C.c_void_p(stream.cuda_stream)


def _check(status: int, where: str):
    if status != MIXKV_OK:
        raise MixkvError(status, where)


def mixkv_workspace_size(p: MixkvParams, n_layers: int) -> int:
    n = C.c_size_t(0)
    _check(lib().mixkv_workspace_size(C.byref(p), n_layers, C.byref(n)), "mixkv_workspace_size")
    return n.value


def alloc_workspace(p: MixkvParams, n_layers: int, device) -> torch.Tensor:
    return torch.empty(mixkv_workspace_size(p, n_layers), dtype=torch.uint8, device=device)


def _ws(workspace: Optional[torch.Tensor]):
    if workspace is None:
        return None, 0
    return C.c_void_p(workspace.data_ptr()), workspace.numel() * workspace.element_size()


def _held(*xs) -> list:
    """The tensors of what a call was prepared over.  Themselves: the call has their addresses, and a program may give a field or a list's place a new one."""
    return [t for x in xs if x is not None for t in
            ([x] if isinstance(x, torch.Tensor) else _held(*vars(x).values()) if is_dataclass(x) else _held(*x) if hasattr(x, "__iter__") else ())]


def mixkv_score(p: MixkvParams, Ks, Vs, Qs, outs: Sequence[LayerOut], workspace: torch.Tensor, stream=None,
                r_given=None, window_lse=None):
    wp, wb = _ws(workspace)
    _check(lib().mixkv_score(C.byref(p), _in_array(Ks, Vs, Qs, r_given, window_lse), _out_array(outs), len(outs), wp, wb, _stream(stream)),
           "mixkv_score")


def mixkv_select(p: MixkvParams, outs: Sequence[LayerOut], workspace: Optional[torch.Tensor] = None, stream=None):
    wp, wb = _ws(workspace)
    _check(lib().mixkv_select(C.byref(p), _out_array(outs), len(outs), wp, wb, _stream(stream)), "mixkv_select")


def mixkv_compress(p: MixkvParams, Ks, Vs, Qs, outs: Sequence[LayerOut], workspace: torch.Tensor, stream=None,
                   r_given=None, window_lse=None):
    wp, wb = _ws(workspace)
    _check(lib().mixkv_compress(C.byref(p), _in_array(Ks, Vs, Qs, r_given, window_lse), _out_array(outs), len(outs), wp, wb,
                                _stream(stream)), "mixkv_compress")


STATIC_SCRATCH_BYTES = 32 << 20


def mixkv_compress_static(p: MixkvParams, Ks, Vs, Qs, outs: Sequence[LayerOut], stream=None, r_given=None, window_lse=None):
    """mixkv_compress on the library's own static workspace (no workspace argument, no allocation)."""
    _check(lib().mixkv_compress_static(C.byref(p), _in_array(Ks, Vs, Qs, r_given, window_lse), _out_array(outs), len(outs),
                                       _stream(stream)), "mixkv_compress_static")


def mixkv_similarity_workspace_size(p: MixkvParams, n_layers: int, block: int) -> int:
    n = C.c_size_t(0)
    _check(lib().mixkv_similarity_workspace_size(C.byref(p), n_layers, block, C.byref(n)),
           "mixkv_similarity_workspace_size")
    return n.value


class PreparedSimilarity:
    """The C argument arrays of one mixkv_similarity call, built once."""

    def __init__(self, p: MixkvParams, Xs, redundancy, block_maps, block: int, workspace: torch.Tensor):
        n = len(Xs)
        self.p, self.n, self.block = p, n, block
        self.ins, self.outs = (MixkvRowsIn * n)(), (MixkvSimilarityOut * n)()
        for i, X in enumerate(Xs):
            assert X.dim() == 4 and X.stride(3) == 1
            self.ins[i] = MixkvRowsIn(X.data_ptr(), X.stride(0), X.stride(1), X.stride(2))
            self.outs[i] = MixkvSimilarityOut(_ptr(None if redundancy is None else redundancy[i]),
                                              _ptr(None if block_maps is None else block_maps[i]))
        self.wp, self.wb = _ws(workspace)
        self._keep = _held(Xs, redundancy, block_maps, workspace)
        self._L = lib()

    def run(self, stream=None):
        _check(self._L.mixkv_similarity(C.byref(self.p), self.ins, self.outs, self.n, self.block, self.wp, self.wb,
                                        _stream(stream)), "mixkv_similarity")


def mixkv_similarity(p: MixkvParams, Xs, block: int, want_map: bool = True, workspace=None, stream=None):
    """Redundancy and (optionally) the block-mean similarity heat-map of every head of the layers Xs
    ([batch, Hkv, N, D] device tensors: keys or values).  Returns (redundancy list, block_map list)."""
    dev = Xs[0].device
    nb = (p.seq_len + block - 1) // block
    red = [torch.empty((p.batch, p.n_kv_heads), dtype=torch.float32, device=dev) for _ in Xs]
    maps = [torch.empty((p.batch, p.n_kv_heads, nb, nb), dtype=torch.float32, device=dev) for _ in Xs] if want_map else None
    if workspace is None:
        workspace = torch.empty(mixkv_similarity_workspace_size(p, len(Xs), block), dtype=torch.uint8, device=dev)
    PreparedSimilarity(p, Xs, red, maps, block, workspace).run(stream)
    return red, maps


class PreparedDecode:
    """The C argument array of one mixkv_decode_attention call, built once.

    caches: per layer a LayerOut as filled by mixkv_compress; tails: per layer (K_tail, V_tail)
    [batch, Hkv, tail_capacity, D] or None; Qs / outs: per layer [batch, Hq, D]."""

    def __init__(self, p: MixkvParams, caches: Sequence[LayerOut], tails, Qs, outs, tail_len: int, workspace="alloc"):
        n = len(caches)
        if isinstance(workspace, str):                # allocate what the shape needs (possibly nothing)
            need = mixkv_decode_workspace_size(p, n, tail_len)
            workspace = torch.empty(need, dtype=torch.uint8, device=Qs[0].device) if need else None
        self.wp, self.wb = _ws(workspace)
        self._ws_keep = workspace
        self.p, self.n, self.tail_len = p, n, tail_len
        self.tail_cap = 0 if tails is None else tails[0][0].shape[2]
        self.arr, self._keep = (MixkvDecodeLayer * n)(), []
        for i, c in enumerate(caches):
            kt, vt = (None, None) if tails is None else tails[i]
            assert Qs[i].is_contiguous() and outs[i].is_contiguous() and (kt is None or kt.is_contiguous())
            self.arr[i] = MixkvDecodeLayer(_ptr(c.K_out), _ptr(c.V_out), _ptr(c.counts), _ptr(c.offsets), _ptr(kt), _ptr(vt),
                                           _ptr(Qs[i]), _ptr(outs[i]))
            self._keep += (c.K_out, c.V_out, c.counts, c.offsets, kt, vt, Qs[i], outs[i])
        self._L = lib()

    def run(self, stream=None):
        _check(self._L.mixkv_decode_attention(C.byref(self.p), self.arr, self.n, self.tail_len, self.tail_cap,
                                              self.wp, self.wb, _stream(stream)), "mixkv_decode_attention")


def mixkv_decode_workspace_size(p: MixkvParams, n_layers: int, tail_len: int) -> int:
    n = C.c_size_t(0)
    _check(lib().mixkv_decode_workspace_size(C.byref(p), n_layers, tail_len, C.byref(n)), "mixkv_decode_workspace_size")
    return n.value


def mixkv_decode_attention(p: MixkvParams, caches, tails, Qs, tail_len: int, stream=None, workspace="alloc"):
    """Returns per layer the attention output [batch, Hq, D] of the new token (dtype of the inputs)."""
    outs = [torch.empty_like(q) for q in Qs]
    PreparedDecode(p, caches, tails, Qs, outs, tail_len, workspace).run(stream)
    return outs


def mixkv_append(p: MixkvParams, new_rows, tails, position: int, stream=None):
    """Copies per layer the new token's (K_new, V_new) [batch, Hkv, D] into row `position` of the
    layer's (K_tail, V_tail) [batch, Hkv, tail_capacity, D], in place."""
    words = []
    for (kn, vn), (kt, vt) in zip(new_rows, tails):
        assert kn.is_contiguous() and vn.is_contiguous() and kt.is_contiguous() and vt.is_contiguous()
        words += (kn.data_ptr(), vn.data_ptr(), kt.data_ptr(), vt.data_ptr())
    n = len(tails)
    _check(lib().mixkv_append(C.byref(p), _structs(MixkvAppendLayer, n, words), n, position, tails[0][0].shape[2], _stream(stream)),
           "mixkv_append")


class PreparedCall:
    """The C argument arrays of one call, built once (so a timed loop measures the library, not ctypes)."""

    def __init__(self, p: MixkvParams, Ks, Vs, Qs, outs: Sequence[LayerOut], workspace: torch.Tensor, r_given=None,
                 window_lse=None):
        self.p, self.n = p, len(outs)
        self.ins, self.outs = _in_array(Ks, Vs, Qs, r_given, window_lse), _out_array(outs)
        self.wp, self.wb = _ws(workspace)
        self._keep = _held(Ks, Vs, Qs, outs, workspace, r_given, window_lse)
        self._L = lib()

    def compress(self, stream=None):
        _check(self._L.mixkv_compress(C.byref(self.p), self.ins, self.outs, self.n, self.wp, self.wb, _stream(stream)),
               "mixkv_compress")

    def compress_profiled(self, stream=None) -> dict:
        ms = (C.c_float * N_STAGES)()
        _check(self._L.mixkv_compress_profiled(C.byref(self.p), self.ins, self.outs, self.n, self.wp, self.wb,
                                               _stream(stream), ms), "mixkv_compress_profiled")
        return {self._L.mixkv_stage_name(i).decode(): float(ms[i]) for i in range(N_STAGES)}

    def score(self, stream=None):
        _check(self._L.mixkv_score(C.byref(self.p), self.ins, self.outs, self.n, self.wp, self.wb, _stream(stream)),
               "mixkv_score")


# ---- the paged cache

def make_paged_params(dtype: str, format: str, batch: int, n_q_heads: int, n_kv_heads: int, head_dim: int, page_rows: int, max_pages: int,
                      n_pages: int, softmax_scale: float = 1.0) -> MixkvPagedParams:
    return MixkvPagedParams(DTYPE[dtype], PAGE_FORMAT[format], batch, n_q_heads, n_kv_heads, head_dim, page_rows, max_pages, n_pages,
                            softmax_scale)


def mixkv_page_bytes(p: MixkvPagedParams) -> int:
    n = C.c_size_t(0)
    _check(lib().mixkv_page_bytes(C.byref(p), C.byref(n)), "mixkv_page_bytes")
    return n.value


@dataclass
class PagedCache:
    """Device tensors of one layer's paged cache."""
    K_pages: Optional[torch.Tensor]              # contiguous, n_pages pages (rows [n_pages, page_rows, D], or bytes in 4 bits)
    V_pages: Optional[torch.Tensor]
    page_table: torch.Tensor                     # [batch, Hkv, max_pages] i32
    lengths: torch.Tensor                        # [batch, Hkv] i32
    K_bounds: Optional[torch.Tensor] = None      # [n_pages, 2, D]


@dataclass
class PagedRows:
    """Dense rows of one layer on their way into pages or out of them (strides like K's for V; an expanded head axis for heads packed
    among one another)."""
    K: torch.Tensor                              # [n_rows, Hkv, D]
    V: torch.Tensor
    row_start: torch.Tensor                      # [batch, Hkv] i32
    row_count: torch.Tensor
    Q: Optional[torch.Tensor] = None             # [n_rows, Hq, D]
    Q_out: Optional[torch.Tensor] = None         # [n_rows, Hq, D] contiguous


@dataclass
class Rope:
    cos: torch.Tensor                            # [n_positions, D / 2] f32
    sin: torch.Tensor
    positions: torch.Tensor                      # [1 or 3, n_rows] i32
    sections: Optional[Sequence[int]] = None     # three of them with three axes


def alloc_paged_cache(p: MixkvPagedParams, device, bounds: bool = False) -> PagedCache:
    """Empty pages, an empty page table (no pages) and lengths of zero, allocated with torch (plumbing for tests and programs)."""
    dt, shape = TORCH_DTYPE[p.dtype], (p.n_pages, p.page_rows, p.head_dim)
    if p.format == PAGE_FORMAT["4bit"]:
        dt, shape = torch.uint8, (p.n_pages, mixkv_page_bytes(p))
    pages = [torch.empty(shape, dtype=dt, device=device) for _ in range(2)]
    return PagedCache(pages[0], pages[1], torch.full((p.batch, p.n_kv_heads, p.max_pages), -1, dtype=torch.int32, device=device),
                      torch.zeros((p.batch, p.n_kv_heads), dtype=torch.int32, device=device),
                      torch.empty((p.n_pages, 2, p.head_dim), dtype=TORCH_DTYPE[p.dtype], device=device) if bounds else None)


def _need(ok: bool, what: str):
    if not ok:
        raise ValueError(what)


def _tensor(t: torch.Tensor, name: str, dtype, shape, device, contiguous=True) -> torch.Tensor:
    """The kernels trust shapes and types: what a pointer does not say is checked here."""
    _need(t.dtype == dtype and tuple(t.shape) == tuple(shape), f"{name}: expected {dtype} {tuple(shape)}, got {t.dtype} {tuple(t.shape)}")
    _need(not contiguous or t.is_contiguous(), f"{name} has to be contiguous")
    _need(t.device == device, f"{name} is on {t.device}, expected {device}")
    return t


def _own(p: MixkvPagedParams) -> MixkvPagedParams:
    """A prepared call's own params: the sizes that its buffers were checked against."""
    return MixkvPagedParams.from_buffer_copy(p)


def _paged_device(caches: Sequence[PagedCache]) -> torch.device:
    _need(len(caches) > 0, "no layers")
    t = caches[0].lengths
    _need(t.is_cuda and t.device.index == torch.cuda.current_device(), "the tensors have to be on the current device")
    return t.device


def _paged_stream(device: torch.device, stream) -> C.c_void_p:
    """The stream of a call prepared on `device`, which has to be the current one then too."""
    current = torch.cuda.current_device()
    _need(current == device.index and (stream is None or stream.device_index == current), "the call was prepared on another device")
    return C.c_void_p(torch._C._cuda_getCurrentRawStream(current) if stream is None else stream.cuda_stream)


def _paged_caches(p: MixkvPagedParams, caches: Sequence[PagedCache], pages: bool, bounds: bool, device):
    units, pool = (p.batch, p.n_kv_heads), 0
    if pages:
        pool = p.n_pages * mixkv_page_bytes(p)
    arr = (MixkvPagedCache * len(caches))()
    for i, c in enumerate(caches):
        _tensor(c.page_table, "page_table", torch.int32, units + (p.max_pages,), device)
        _tensor(c.lengths, "lengths", torch.int32, units, device)
        if pages:
            for name, t in (("K_pages", c.K_pages), ("V_pages", c.V_pages)):
                _need(t is not None and t.is_contiguous() and t.device == device and t.numel() * t.element_size() == pool,
                      f"{name} has to be {pool} contiguous bytes on {device}")
        _need(c.K_bounds is not None or not bounds, "K_bounds is needed")
        if c.K_bounds is not None:
            _tensor(c.K_bounds, "K_bounds", TORCH_DTYPE[p.dtype], (p.n_pages, 2, p.head_dim), device)
        arr[i] = MixkvPagedCache(_ptr(c.K_pages), _ptr(c.V_pages), _ptr(c.K_bounds), _ptr(c.page_table), _ptr(c.lengths))
    return arr


def _paged_rows(p: MixkvPagedParams, rows: Sequence[PagedRows], queries: bool, device):
    arr, n_rows, dt = (MixkvPagedRows * len(rows))(), rows[0].K.shape[0], TORCH_DTYPE[p.dtype]
    for i, r in enumerate(rows):
        shape = (n_rows, p.n_kv_heads, p.head_dim)
        for name, t in (("K", r.K), ("V", r.V)):
            _tensor(t, name, dt, shape, device, contiguous=False)
            _need(t.stride(2) == 1 and t.stride() == r.K.stride(), "K and V need the same strides, the last one 1")
        for name, t in (("row_start", r.row_start), ("row_count", r.row_count)):
            _tensor(t, name, torch.int32, (p.batch, p.n_kv_heads), device)
        q, qs = (r.Q, r.Q_out) if queries else (None, None)
        if q is not None:
            _tensor(q, "Q", dt, (n_rows, p.n_q_heads, p.head_dim), device, contiguous=False)
            _need(q.stride(2) == 1 and qs is not None, "Q needs stride 1 along a row, and Q_out")
            _tensor(qs, "Q_out", dt, (n_rows, p.n_q_heads, p.head_dim), device)
        st = (0, 0) if q is None else (q.stride(0), q.stride(1))
        arr[i] = MixkvPagedRows(_ptr(r.K), _ptr(r.V), r.K.stride(0), r.K.stride(1), _ptr(r.row_start), _ptr(r.row_count), _ptr(q), *st, _ptr(qs))
    return arr, n_rows


class PreparedPagedAppend:
    """The C arguments of one mixkv_paged_append call, built once over buffers that a serving loop keeps (a workspace that a prepared call allocates is
    the current stream's: a run on another stream has to wait for that one, as for any tensor).  The call is about the tensors that it was prepared over, and holds
    them: after a field has got another one, prepare again.  `max_count`: the largest row_count as far as the host knows it (None: the dense tensor's rows)."""

    def __init__(self, p: MixkvPagedParams, caches: Sequence[PagedCache], rows: Sequence[PagedRows], rope: Optional[Rope] = None,
                 max_count: Optional[int] = None):
        self.device = device = _paged_device(caches)
        _need(len(caches) == len(rows), "a rows entry for every cache")
        self.p, self.n, self.caches = _own(p), len(caches), _paged_caches(p, caches, True, False, device)
        self.rows, self.n_rows = _paged_rows(p, rows, True, device)
        self.max_count, self.rope = self.n_rows if max_count is None else max_count, None
        if rope is not None:
            half, axes = p.head_dim // 2, rope.positions.shape[0]
            for name, t in (("cos", rope.cos), ("sin", rope.sin)):
                _tensor(t, name, torch.float32, (rope.cos.shape[0], half), device)
            _tensor(rope.positions, "positions", torch.int32, (axes, self.n_rows), device)
            _need(axes != 3 or rope.sections is not None and len(rope.sections) == 3, "three axes need three sections")
            self.rope = MixkvRope(_ptr(rope.cos), _ptr(rope.sin), rope.cos.shape[0], _ptr(rope.positions), axes,
                                  (C.c_int32 * 3)(*(rope.sections if axes == 3 else (0, 0, 0))))
        self._keep = _held(caches, rows, rope)
        self._args = (C.byref(self.p), self.caches, self.rows, self.n, None if self.rope is None else C.byref(self.rope), self.n_rows,
                      self.max_count)
        self._call = lib().mixkv_paged_append

    def run(self, stream=None):
        _check(self._call(*self._args, _paged_stream(self.device, stream)), "mixkv_paged_append")


def mixkv_paged_append(p: MixkvPagedParams, caches: Sequence[PagedCache], rows: Sequence[PagedRows], rope: Optional[Rope] = None,
                       max_count: Optional[int] = None, stream=None):
    """Rows into pages, in place (with rows[i].Q: the rotated queries into rows[i].Q_out)."""
    PreparedPagedAppend(p, caches, rows, rope, max_count).run(stream)


class PreparedPagedRead:
    """The C arguments of one mixkv_paged_read call: rows[i].K and .V receive the newest row_count rows of every head."""

    def __init__(self, p: MixkvPagedParams, caches: Sequence[PagedCache], rows: Sequence[PagedRows], max_count: Optional[int] = None):
        self.device = device = _paged_device(caches)
        _need(len(caches) == len(rows), "a rows entry for every cache")
        self.p, self.n, self.caches = _own(p), len(caches), _paged_caches(p, caches, True, False, device)
        self.rows, self.n_rows = _paged_rows(p, rows, False, device)
        self.max_count = self.n_rows if max_count is None else max_count
        self._keep = _held(caches, rows)
        self._args = (C.byref(self.p), self.caches, self.rows, self.n, self.n_rows, self.max_count)
        self._call = lib().mixkv_paged_read

    def run(self, stream=None):
        _check(self._call(*self._args, _paged_stream(self.device, stream)), "mixkv_paged_read")


def mixkv_paged_read(p: MixkvPagedParams, caches: Sequence[PagedCache], rows: Sequence[PagedRows], max_count: Optional[int] = None, stream=None):
    PreparedPagedRead(p, caches, rows, max_count).run(stream)


def _paged_workspace(workspace, need: int, device):
    if isinstance(workspace, str):                    # allocate what the shape needs (possibly nothing)
        return torch.empty(need, dtype=torch.uint8, device=device) if need else None
    _need(workspace is None or workspace.is_contiguous() and workspace.device == device, f"the workspace has to be contiguous, on {device}")
    return workspace


def mixkv_paged_select_workspace_size(p: MixkvPagedParams, n_layers: int) -> int:
    n = C.c_size_t(0)
    _check(lib().mixkv_paged_select_workspace_size(C.byref(p), n_layers, C.byref(n)), "mixkv_paged_select_workspace_size")
    return n.value


class PreparedPagedSelect:
    """The C arguments of one mixkv_paged_select call.  Qs: per layer [batch, Hq, D]; selected [batch, Hkv, max_selected] and n_selected
    [batch, Hkv] i32 receive the places of the selected pages."""

    def __init__(self, p: MixkvPagedParams, caches: Sequence[PagedCache], Qs, selected, n_selected, keep_first: int = 1, keep_last: int = 1,
                 workspace="alloc"):
        self.device = device = _paged_device(caches)
        n = len(caches)
        _need(n == len(Qs) == len(selected) == len(n_selected), "queries and selections for every cache")
        self.p, self.n, self.caches, self.most = _own(p), n, _paged_caches(p, caches, False, True, device), selected[0].shape[-1]
        self.arr = (MixkvPagedSelectLayer * n)()
        for i in range(n):
            _tensor(Qs[i], "Q", TORCH_DTYPE[p.dtype], (p.batch, p.n_q_heads, p.head_dim), device)
            _tensor(selected[i], "selected", torch.int32, (p.batch, p.n_kv_heads, self.most), device)
            _tensor(n_selected[i], "n_selected", torch.int32, (p.batch, p.n_kv_heads), device)
            self.arr[i] = MixkvPagedSelectLayer(_ptr(Qs[i]), _ptr(selected[i]), _ptr(n_selected[i]))
        self.first, self.last = keep_first, keep_last
        workspace = _paged_workspace(workspace, mixkv_paged_select_workspace_size(p, n) if isinstance(workspace, str) else 0, device)
        self.wp, self.wb = _ws(workspace)
        self._keep = _held(caches, Qs, selected, n_selected, workspace)
        self._args = (C.byref(self.p), self.caches, self.arr, self.n, self.most, self.first, self.last, self.wp, self.wb)
        self._call = lib().mixkv_paged_select

    def run(self, stream=None):
        _check(self._call(*self._args, _paged_stream(self.device, stream)), "mixkv_paged_select")


def mixkv_paged_select(p: MixkvPagedParams, caches: Sequence[PagedCache], Qs, max_selected: int, keep_first: int = 1, keep_last: int = 1,
                       workspace="alloc", stream=None):
    """Returns per layer the places of the selected pages [batch, Hkv, max_selected] and their numbers [batch, Hkv], allocated on the call's stream."""
    dev, n = _paged_device(caches), len(caches)
    with torch.cuda.stream(stream):                   # what is allocated here is the stream's (None: the current one's)
        selected = [torch.empty((p.batch, p.n_kv_heads, max_selected), dtype=torch.int32, device=dev) for _ in range(n)]
        n_selected = [torch.empty((p.batch, p.n_kv_heads), dtype=torch.int32, device=dev) for _ in range(n)]
        PreparedPagedSelect(p, caches, Qs, selected, n_selected, keep_first, keep_last, workspace).run(stream)
    return selected, n_selected


def mixkv_paged_attention_workspace_size(p: MixkvPagedParams, n_layers: int, max_rows: int) -> int:
    n = C.c_size_t(0)
    _check(lib().mixkv_paged_attention_workspace_size(C.byref(p), n_layers, max_rows, C.byref(n)), "mixkv_paged_attention_workspace_size")
    return n.value


class PreparedPagedAttention:
    """The C arguments of one mixkv_paged_attention call.  Qs / outs: per layer [batch, Hq, D]; selected / n_selected: per layer the places
    of the pages to attend to, or None for all; max_rows: the largest number of rows of a head as far as the host knows it (None:
    what the page table, or the selection, can hold)."""

    def __init__(self, p: MixkvPagedParams, caches: Sequence[PagedCache], Qs, outs, selected=None, n_selected=None,
                 max_rows: Optional[int] = None, workspace="alloc"):
        self.device = device = _paged_device(caches)
        n, sparse = len(caches), selected is not None
        _need(n == len(Qs) == len(outs) and (not sparse or n == len(selected) == len(n_selected)), "queries, outputs and selections for every cache")
        self.p, self.n, self.caches = _own(p), n, _paged_caches(p, caches, True, False, device)
        self.most = selected[0].shape[-1] if sparse else 0
        self.rows = max_rows if max_rows is not None else (min(self.most, p.max_pages) if sparse else p.max_pages) * p.page_rows
        self.arr = (MixkvPagedAttentionLayer * n)()
        for i in range(n):
            for name, t in (("Q", Qs[i]), ("out", outs[i])):
                _tensor(t, name, TORCH_DTYPE[p.dtype], (p.batch, p.n_q_heads, p.head_dim), device)
            if sparse:
                _tensor(selected[i], "selected", torch.int32, (p.batch, p.n_kv_heads, self.most), device)
                _tensor(n_selected[i], "n_selected", torch.int32, (p.batch, p.n_kv_heads), device)
            self.arr[i] = MixkvPagedAttentionLayer(_ptr(Qs[i]), _ptr(outs[i]), *((_ptr(selected[i]), _ptr(n_selected[i])) if sparse else (None, None)))
        need = mixkv_paged_attention_workspace_size(p, n, self.rows) if isinstance(workspace, str) else 0
        workspace = _paged_workspace(workspace, need, device)
        self.wp, self.wb = _ws(workspace)
        self._keep = _held(caches, Qs, outs, selected, n_selected, workspace)
        self._args = (C.byref(self.p), self.caches, self.arr, self.n, self.most, self.rows, self.wp, self.wb)
        self._call = lib().mixkv_paged_attention

    def run(self, stream=None):
        _check(self._call(*self._args, _paged_stream(self.device, stream)), "mixkv_paged_attention")


def mixkv_paged_attention(p: MixkvPagedParams, caches: Sequence[PagedCache], Qs, selected=None, n_selected=None, max_rows: Optional[int] = None,
                          workspace="alloc", stream=None):
    """Returns per layer the attention output [batch, Hq, D] of the new token of every sequence, allocated on the call's stream."""
    _paged_device(caches)
    with torch.cuda.stream(stream):                   # what is allocated here is the stream's (None: the current one's)
        outs = [torch.empty_like(q) for q in Qs]
        PreparedPagedAttention(p, caches, Qs, outs, selected, n_selected, max_rows, workspace).run(stream)
    return outs


@dataclass
class PagedQueries:
    """One layer's queries of new rows, as mixkv_paged_append rotated them, and what the attention makes of them."""
    Q: torch.Tensor                              # [n_rows, Hq, D], stride 1 along D
    row_start: torch.Tensor                      # [batch, Hkv] i32
    row_count: torch.Tensor
    out: Optional[torch.Tensor] = None           # [n_rows, Hq, D] contiguous (attention)
    lse: Optional[torch.Tensor] = None           # [n_rows, Hq] f32 contiguous (attention: if wanted; weights: needed)


EVERY_ROW = 1 << 30                              # a window that leaves nothing out


def _paged_queries(p: MixkvPagedParams, queries: Sequence[PagedQueries], attention: bool, device):
    arr, n_rows, dt = (MixkvPagedQueries * len(queries))(), queries[0].Q.shape[0], TORCH_DTYPE[p.dtype]
    for i, q in enumerate(queries):
        shape = (n_rows, p.n_q_heads, p.head_dim)
        _tensor(q.Q, "Q", dt, shape, device, contiguous=False)
        _need(q.Q.stride(2) == 1, "Q needs stride 1 along a row")
        for name, t in (("row_start", q.row_start), ("row_count", q.row_count)):
            _tensor(t, name, torch.int32, (p.batch, p.n_kv_heads), device)
        _need(q.out is not None if attention else q.lse is not None, "out is needed" if attention else "lse is needed")
        if attention:
            _tensor(q.out, "out", dt, shape, device)
        if q.lse is not None:
            _tensor(q.lse, "lse", torch.float32, shape[:2], device)
        arr[i] = MixkvPagedQueries(_ptr(q.Q), q.Q.stride(0), q.Q.stride(1), _ptr(q.row_start), _ptr(q.row_count), _ptr(q.out), _ptr(q.lse))
    return arr, n_rows


def mixkv_paged_window_attention_workspace_size(p: MixkvPagedParams, n_layers: int, n_rows: int, window: int, keep_first: int, max_count: int,
                                                max_rows: int) -> int:
    n = C.c_size_t(0)
    _check(lib().mixkv_paged_window_attention_workspace_size(C.byref(p), n_layers, n_rows, window, keep_first, max_count, max_rows, C.byref(n)),
           "mixkv_paged_window_attention_workspace_size")
    return n.value


def mixkv_paged_weights_workspace_size(p: MixkvPagedParams, n_layers: int, n_rows: int, window: int, keep_first: int, max_count: int, max_rows: int) -> int:
    n = C.c_size_t(0)
    _check(lib().mixkv_paged_weights_workspace_size(C.byref(p), n_layers, n_rows, window, keep_first, max_count, max_rows, C.byref(n)),
           "mixkv_paged_weights_workspace_size")
    return n.value


class PreparedPagedWindowAttention:
    """The C arguments of one mixkv_paged_window_attention call.  queries: per layer a PagedQueries with `out` (and `lse`, if wanted); max_count: the
    largest row_count, a bound that is kept to (None: the queries' rows); max_rows: the largest length as far as the host knows it (None: what the page table can hold)."""

    def __init__(self, p: MixkvPagedParams, caches: Sequence[PagedCache], queries: Sequence[PagedQueries], window: int = EVERY_ROW, keep_first: int = 0,
                 max_count: Optional[int] = None, max_rows: Optional[int] = None, workspace="alloc"):
        self.device = device = _paged_device(caches)
        _need(len(caches) == len(queries), "queries for every cache")
        self.p, self.n, self.caches = _own(p), len(caches), _paged_caches(p, caches, True, False, device)
        self.queries, n_rows = _paged_queries(p, queries, True, device)
        sizes = (n_rows, window, keep_first, n_rows if max_count is None else max_count, p.max_pages * p.page_rows if max_rows is None else max_rows)
        workspace = _paged_workspace(workspace, mixkv_paged_window_attention_workspace_size(p, self.n, *sizes) if isinstance(workspace, str) else 0, device)
        self.wp, self.wb = _ws(workspace)
        self._keep = _held(caches, queries, workspace)
        self._args = (C.byref(self.p), self.caches, self.queries, self.n, *sizes, self.wp, self.wb)
        self._call = lib().mixkv_paged_window_attention

    def run(self, stream=None):
        _check(self._call(*self._args, _paged_stream(self.device, stream)), "mixkv_paged_window_attention")


def mixkv_paged_window_attention(p: MixkvPagedParams, caches: Sequence[PagedCache], queries: Sequence[PagedQueries], window: int = EVERY_ROW, keep_first: int = 0,
                                 max_count: Optional[int] = None, max_rows: Optional[int] = None, workspace="alloc", stream=None):
    """Attention of the new rows into queries[i].out (and .lse)."""
    with torch.cuda.stream(stream):                   # what is allocated here is the stream's (None: the current one's)
        PreparedPagedWindowAttention(p, caches, queries, window, keep_first, max_count, max_rows, workspace).run(stream)


def _weight_pool(p: MixkvPagedParams, t: torch.Tensor, name: str, device) -> torch.Tensor:
    return _tensor(t, name, torch.float32, (p.n_pages, p.page_rows), device)


class PreparedPagedWeights:
    """The C arguments of one mixkv_paged_weights call.  queries: per layer a PagedQueries with the `lse` of the attention; weights: per layer
    [n_pages, page_rows] f32, raised in place (a page is listed for one place of one head)."""

    def __init__(self, p: MixkvPagedParams, caches: Sequence[PagedCache], queries: Sequence[PagedQueries], weights: Sequence[torch.Tensor],
                 window: int = EVERY_ROW, keep_first: int = 0, max_count: Optional[int] = None, max_rows: Optional[int] = None, workspace="alloc"):
        self.device = device = _paged_device(caches)
        _need(len(caches) == len(queries) == len(weights), "queries and weights for every cache")
        self.p, self.n, self.caches = _own(p), len(caches), _paged_caches(p, caches, False, False, device)
        _key_pages(p, caches, device)
        self.queries, n_rows = _paged_queries(p, queries, False, device)
        self.weights = (C.c_void_p * self.n)(*(_weight_pool(p, w, "weights", device).data_ptr() for w in weights))
        sizes = (n_rows, window, keep_first, n_rows if max_count is None else max_count, p.max_pages * p.page_rows if max_rows is None else max_rows)
        workspace = _paged_workspace(workspace, mixkv_paged_weights_workspace_size(p, self.n, *sizes) if isinstance(workspace, str) else 0, device)
        self.wp, self.wb = _ws(workspace)
        self._keep = _held(caches, queries, weights, workspace)
        self._args = (C.byref(self.p), self.caches, self.queries, self.weights, self.n, *sizes, self.wp, self.wb)
        self._call = lib().mixkv_paged_weights

    def run(self, stream=None):
        _check(self._call(*self._args, _paged_stream(self.device, stream)), "mixkv_paged_weights")


def _key_pages(p: MixkvPagedParams, caches: Sequence[PagedCache], device):
    pool = p.n_pages * mixkv_page_bytes(p)
    for c in caches:
        t = c.K_pages
        _need(t is not None and t.is_contiguous() and t.device == device and t.numel() * t.element_size() == pool, f"K_pages has to be {pool} contiguous bytes on {device}")


def mixkv_paged_weights(p: MixkvPagedParams, caches: Sequence[PagedCache], queries: Sequence[PagedQueries], weights: Sequence[torch.Tensor],
                        window: int = EVERY_ROW, keep_first: int = 0, max_count: Optional[int] = None, max_rows: Optional[int] = None, workspace="alloc",
                        stream=None):
    """The weights that the new rows give to the cached ones, added to `weights` in place."""
    with torch.cuda.stream(stream):                   # what is allocated here is the stream's (None: the current one's)
        PreparedPagedWeights(p, caches, queries, weights, window, keep_first, max_count, max_rows, workspace).run(stream)


def mixkv_paged_evict_workspace_size(p: MixkvPagedParams, n_layers: int, max_rows: int) -> int:
    n = C.c_size_t(0)
    _check(lib().mixkv_paged_evict_workspace_size(C.byref(p), n_layers, max_rows, C.byref(n)), "mixkv_paged_evict_workspace_size")
    return n.value


class PreparedPagedEvict:
    """The C arguments of one mixkv_paged_evict call.  into: per layer the cache that the kept rows go to (pools of the same size, the caches' own or others; its
    page_table lists free pages, its lengths are written); weights, weights_into: [n_pages, page_rows] f32 of the one's and the other's pages; keep: per layer
    [batch, Hkv] i32; kept: [batch, Hkv, max_keep] i32 receives the places that the rows come from."""

    def __init__(self, p: MixkvPagedParams, caches: Sequence[PagedCache], into: Sequence[PagedCache], weights: Sequence[torch.Tensor], keep, kept,
                 keep_first: int = 0, keep_last: int = 0, weights_into: Optional[Sequence[torch.Tensor]] = None, max_rows: Optional[int] = None, workspace="alloc"):
        self.device = device = _paged_device(caches)
        n = len(caches)
        _need(n == len(into) == len(weights) == len(keep) == len(kept) and (weights_into is None or n == len(weights_into)), "one of each for every cache")
        self.p, self.n, self.caches, self.into = _own(p), n, _paged_caches(p, caches, True, False, device), _paged_caches(p, into, True, False, device)
        most = kept[0].shape[-1]
        self.arr = (MixkvPagedEvictLayer * n)()
        for i in range(n):
            _weight_pool(p, weights[i], "weights", device)
            if weights_into is not None:
                _weight_pool(p, weights_into[i], "weights_into", device)
            _tensor(keep[i], "keep", torch.int32, (p.batch, p.n_kv_heads), device)
            _tensor(kept[i], "kept", torch.int32, (p.batch, p.n_kv_heads, most), device)
            self.arr[i] = MixkvPagedEvictLayer(_ptr(weights[i]), _ptr(None if weights_into is None else weights_into[i]), _ptr(keep[i]), _ptr(kept[i]),
                                               _ptr(into[i].lengths))
        rows = p.max_pages * p.page_rows if max_rows is None else max_rows
        workspace = _paged_workspace(workspace, mixkv_paged_evict_workspace_size(p, n, rows) if isinstance(workspace, str) else 0, device)
        self.wp, self.wb = _ws(workspace)
        self._keep = _held(caches, into, weights, weights_into, keep, kept, workspace)
        self._args = (C.byref(self.p), self.caches, self.into, self.arr, n, most, keep_first, keep_last, rows, self.wp, self.wb)
        self._call = lib().mixkv_paged_evict

    def run(self, stream=None):
        _check(self._call(*self._args, _paged_stream(self.device, stream)), "mixkv_paged_evict")


def mixkv_paged_evict(p: MixkvPagedParams, caches: Sequence[PagedCache], into: Sequence[PagedCache], weights: Sequence[torch.Tensor], keep, max_keep: int,
                      keep_first: int = 0, keep_last: int = 0, weights_into: Optional[Sequence[torch.Tensor]] = None, max_rows: Optional[int] = None,
                      workspace="alloc", stream=None):
    """Moves what is kept into the pages of `into`; returns per layer the places [batch, Hkv, max_keep] that the rows come from, allocated on the call's stream."""
    dev = _paged_device(caches)
    with torch.cuda.stream(stream):                   # what is allocated here is the stream's (None: the current one's)
        kept = [torch.empty((p.batch, p.n_kv_heads, max_keep), dtype=torch.int32, device=dev) for _ in caches]
        PreparedPagedEvict(p, caches, into, weights, keep, kept, keep_first, keep_last, weights_into, max_rows, workspace).run(stream)
    return kept


def compacted_rows(p: MixkvParams, out: LayerOut) -> PagedRows:
    """What mixkv_compress left of one layer, as dense rows for mixkv_paged_append (its counts are the lengths): no copies of rows."""
    bt, h, d = p.batch, p.n_kv_heads, p.head_dim
    first = torch.arange(bt, dtype=torch.int32, device=out.counts.device)[:, None] * (h * p.budget)
    if p.budget_mode == BUDGET_MODE["fixed"]:
        start = first + torch.arange(h, dtype=torch.int32, device=out.counts.device) * p.budget
    else:
        start = first + out.offsets[:, :h]
    K, V = (t.view(-1, 1, d).expand(-1, h, -1) for t in (out.K_out, out.V_out))
    return PagedRows(K, V, start.contiguous(), out.counts.contiguous())
