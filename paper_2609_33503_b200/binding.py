"""Python binding of the RelaxKV C ABI (include/relaxkv.h): argument marshalling only.

Every function here has the name of the C entry point it calls and does nothing but turn torch
tensors and Python lists into pointers and sizes.  All computation runs in the CUDA kernels of
librelaxkv.so; there is no CPU path and no fallback: if the library has not been built, loading
fails with an error.
"""
from __future__ import annotations

import ctypes
import operator
import os
from typing import List, Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "librelaxkv.so")

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED_SHAPE, ERR_WORKSPACE_TOO_SMALL, ERR_CUDA, ERR_BAD_INDEX, ERR_TIMEOUT = range(7)
CTX_UNION, CTX_FULL_PREFIX = 0, 1

ENTRY_POINTS = (
    "relaxkv_status_string", "relaxkv_anchor_count", "relaxkv_workspace_bytes", "relaxkv_score_select",
    "relaxkv_build_active_sets", "relaxkv_sparse_ctx_attention", "relaxkv_scatter_kv", "relaxkv_gather_kv",
    "relaxkv_sparse_ctx_attention_simt", "relaxkv_read_device_status", "relaxkv_select_topk",
    "relaxkv_build_active_sets_static", "relaxkv_debug_wait_timeout",
    "relaxkv_list_attention", "relaxkv_cache_attention",
    "relaxkv_scatter_kv_lists", "relaxkv_mean_scores", "relaxkv_scale_scores", "relaxkv_query_prefill_attention", "relaxkv_rmsnorm", "relaxkv_linear", "relaxkv_linear_qkv", "relaxkv_linear_swiglu", "relaxkv_rope", "relaxkv_qk_norm_rope", "relaxkv_qk_norm_rope_append",
    "relaxkv_swiglu", "relaxkv_target_positions", "relaxkv_carry_rows", "relaxkv_set_chained_launch",
    "relaxkv_continuation_workspace_bytes", "relaxkv_build_block_tables", "relaxkv_qk_norm_rope_append_paged", "relaxkv_shared_prefix_attention",
    "relaxkv_block_bounds", "relaxkv_select_blocks", "relaxkv_block_sparse_attention",
    "relaxkv_rotary_frequencies", "relaxkv_qk_norm_rotate", "relaxkv_append_quantized", "relaxkv_read_quantized",
    "relaxkv_quantized_workspace_bytes", "relaxkv_quantized_attention",
)


class RelaxKVError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status})")


class _Tuning(ctypes.Structure):
    _fields_ = [("attention_ctx_splits", ctypes.c_int32), ("attention_persistent", ctypes.c_int32),
                ("attention_grid_blocks", ctypes.c_int32)]


class _Shape(ctypes.Structure):
    _fields_ = [("n_req", ctypes.c_int32), ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("h_ctx_len", ctypes.POINTER(ctypes.c_int32)),
                ("h_q_len", ctypes.POINTER(ctypes.c_int32)), ("softmax_scale", ctypes.c_float),
                ("h_tuning", ctypes.POINTER(_Tuning))]


class _CacheView(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("token_stride", ctypes.c_int64),
                ("head_stride", ctypes.c_int64), ("h_req_token_offset", ctypes.POINTER(ctypes.c_int64))]


class _PagedCache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("block_stride", ctypes.c_int64), ("token_stride", ctypes.c_int64),
                ("head_stride", ctypes.c_int64), ("block_size", ctypes.c_int32), ("n_blocks", ctypes.c_int32)]


class _QuantizedCache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_exp", ctypes.c_void_p), ("v_exp", ctypes.c_void_p),
                ("block_stride", ctypes.c_int64), ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64), ("block_size", ctypes.c_int32),
                ("n_blocks", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("type", ctypes.c_int32)]


class _Rotary(ctypes.Structure):
    _fields_ = [("freq", ctypes.c_void_p), ("dims", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("amplitude", ctypes.c_float)]


class _ContinuationRows(ctypes.Structure):
    _fields_ = [("n_seq", ctypes.c_int32), ("table_width", ctypes.c_int32), ("table_stride", ctypes.c_int64), ("n_rows", ctypes.c_int64),
                ("max_len", ctypes.c_int32), ("h_seq_cu", ctypes.c_void_p), ("h_max_rows", ctypes.c_void_p), ("row_cu", ctypes.c_void_p),
                ("row_seq", ctypes.c_void_p), ("row_len", ctypes.c_void_p), ("block_table", ctypes.c_void_p)]


# Argument types of the entry points, declared once so that a call passes plain integers and floats (p pointer or stream,
# i int32, l int64, z size_t, f float, d double): a ctypes object per argument and a stream object per call were most of
# the 15 us that a call of a decode step took on the host.
_CTYPE = {"p": ctypes.c_void_p, "i": ctypes.c_int32, "l": ctypes.c_int64, "z": ctypes.c_size_t, "f": ctypes.c_float, "d": ctypes.c_double}
_ST = ctypes.c_int32
_SIGNATURES = {
    "relaxkv_status_string": (ctypes.c_char_p, "i"), "relaxkv_anchor_count": (ctypes.c_int32, "id"),
    "relaxkv_workspace_bytes": (ctypes.c_size_t, "pip"), "relaxkv_set_chained_launch": (ctypes.c_int32, "i"),
    "relaxkv_score_select": (_ST, "pi pp pp ppp pzp"), "relaxkv_select_topk": (_ST, "pip ppp p"),
    "relaxkv_build_active_sets": (_ST, "pipp pppppp p pzp"), "relaxkv_build_active_sets_static": (_ST, "pipp pppppp p p"),
    "relaxkv_sparse_ctx_attention": (_ST, "pip ppp pppp lpp pp pzp"),
    "relaxkv_sparse_ctx_attention_simt": (_ST, "pip ppp pppp lpp pp pzp"),
    "relaxkv_scatter_kv": (_ST, "pp pp pppp p p"), "relaxkv_gather_kv": (_ST, "pip pp pppp p pp lp"),
    "relaxkv_list_attention": (_ST, "pp ppp pppp lpp pp pzp"), "relaxkv_cache_attention": (_ST, "pp p pp lp pp pzp"),
    "relaxkv_scatter_kv_lists": (_ST, "pp pp pp p p"), "relaxkv_mean_scores": (_ST, "pi pp p"),
    "relaxkv_scale_scores": (_ST, "pi pf p"), "relaxkv_query_prefill_attention": (_ST, "pp ppp p pzp"),
    "relaxkv_rmsnorm": (_ST, "ppp li f p"), "relaxkv_linear": (_ST, "pppp lii p"), "relaxkv_linear_qkv": (_ST, "pp ppp liii p"),
    "relaxkv_linear_swiglu": (_ST, "ppp lii p"), "relaxkv_rope": (_ST, "p lii p f p"),
    "relaxkv_qk_norm_rope": (_ST, "pp liii pp f p f p"),
    "relaxkv_qk_norm_rope_append": (_ST, "pp ppp l pp f ppp f p"), "relaxkv_swiglu": (_ST, "pp li p"),
    "relaxkv_target_positions": (_ST, "p pppp p p p"), "relaxkv_carry_rows": (_ST, "p pp i ppp p p"),
    "relaxkv_continuation_workspace_bytes": (ctypes.c_size_t, "pli"),
    "relaxkv_build_block_tables": (_ST, "ii pppp i pp i ll pp ppppp p"),
    "relaxkv_qk_norm_rope_append_paged": (_ST, "p ppp liii pp f pp f pp"),
    "relaxkv_shared_prefix_attention": (_ST, "pppp ppp pzp"), "relaxkv_block_bounds": (_ST, "pp i pp p"),
    "relaxkv_select_blocks": (_ST, "p i pp pp iii p pzp"), "relaxkv_block_sparse_attention": (_ST, "pppp ipi ppp pzp"),
    "relaxkv_rotary_frequencies": (_ST, "id id i dd pp"), "relaxkv_qk_norm_rotate": (_ST, "ppll ppll liii pp f pp p"),
    "relaxkv_append_quantized": (_ST, "p ppll ppll liii pp f pp p p"), "relaxkv_read_quantized": (_ST, "pp lii pp pp ll p"),
    "relaxkv_quantized_workspace_bytes": (ctypes.c_size_t, "iii"), "relaxkv_quantized_attention": (_ST, "pp iii f ppp pzp"),
    "relaxkv_debug_wait_timeout": (_ST, "p"), "relaxkv_read_device_status": (_ST, "pp p"),
}

_lib = None


def _native():
    """The module of csrc/py_calls.cpp: arguments and calls in native code."""
    try:
        from . import _calls
    except ImportError as e:
        raise RuntimeError(f"{os.path.join(_HERE, '_calls.so')} is missing or cannot be loaded ({e}): build it with "
                           "`python -m paper_2609_33503_b200.build`") from e
    return _calls


def lib() -> ctypes.CDLL:
    """The loaded C-ABI library.  Raises if it has not been built (no fallback exists)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2609_33503_b200.build` "
                               "(nvcc, sm_100a). There is no CPU fallback.")
        l = ctypes.CDLL(LIB_PATH)
        for name, (restype, args) in _SIGNATURES.items():
            fn = getattr(l, name)
            fn.restype, fn.argtypes = restype, [_CTYPE[c] for c in args.replace(" ", "")]
            setattr(l, name, _native().bind(name, ctypes.cast(fn, ctypes.c_void_p).value, fn))
        _lib = l
    return _lib


def status_string(status: int) -> str:
    return lib().relaxkv_status_string(int(status)).decode()


def relaxkv_set_chained_launch(on: bool) -> bool:
    """Chained (programmatic dependent) launches of the short kernels on or off, process-wide; returns the previous
    setting."""
    return bool(lib().relaxkv_set_chained_launch(1 if on else 0))


def _check(status: int, where: str) -> None:
    if status != OK:
        raise RelaxKVError(status, where)


_i32_types = {}                    # array types by length: making one is most of what a short array costs


def _i32(xs: Optional[Sequence[int]]):
    if xs is None:
        return None
    n = len(xs)
    kind = _i32_types.get(n)
    if kind is None:
        kind = ctypes.c_int32 * n
        if n <= 64:                # (the most requests of a call; longer lists are refused by the library)
            _i32_types[n] = kind
    return kind(*map(int, xs))


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _args(codes: str, *args):
    """The arguments of an entry point as its bound form takes them, one code each: p a tensor (or None), h host integers (or None), s a
    ctypes structure, . a plain value.  # is a number of elements, not passed on: I, W, F and C behind it are tensors of int32, bfloat16, float32
    or int8 that have to hold as many (ValueError); i, w, f and c have to be contiguous whatever their size.  The first call puts the native
    function in this one's place."""
    global _args
    _args = _native().marshal
    return _args(codes, *args)


class Offsets:
    """Offsets inside a tensor that the caller keeps, in the place of the slice that starts there: a slice costs the host 1 to 3 us, as
    much as marshalling the rest of a call.  (A plain number is not taken for an address.)"""

    __slots__ = ("_address",)

    def __init__(self, tensor: torch.Tensor, first: int):
        self._address = tensor.data_ptr() + tensor.element_size() * first

    def data_ptr(self) -> int:
        return self._address


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)     # the handle without a Stream object around it
_current_device = getattr(torch._C, "_cuda_getDevice", None)
_raw_synchronize = getattr(torch._C, "_cuda_synchronize", None)


def synchronize(device: torch.device) -> None:
    """torch.cuda.synchronize; without its change of device where the device is the current one."""
    if (_raw_synchronize is not None and _current_device is not None and device.type == "cuda" and torch.cuda.is_initialized()
            and (device.index is None or device.index == _current_device())):
        _raw_synchronize()
    else:
        torch.cuda.synchronize(device)


def _stream(stream) -> int:
    if stream is None:
        if _raw_stream is not None and _current_device is not None and torch.cuda.is_initialized():
            return _raw_stream(_current_device())
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


class Shape:
    """Host-side relaxkv_shape; keeps its arrays alive."""

    def __init__(self, n_q_heads: int, n_kv_heads: int, head_dim: int, ctx_lens: Sequence[int],
                 q_lens: Optional[Sequence[int]] = None, softmax_scale: Optional[float] = None,
                 attention_ctx_splits: int = 0, attention_persistent: int = 0, attention_grid_blocks: int = 0):
        self.ctx_lens = [int(x) for x in ctx_lens]
        self.q_lens = None if q_lens is None else [int(x) for x in q_lens]
        self._ctx = _i32(self.ctx_lens)
        self._q = _i32(self.q_lens)
        self.c = _Shape()
        self.c.n_req = len(self.ctx_lens)
        self.c.n_q_heads, self.c.n_kv_heads, self.c.head_dim = int(n_q_heads), int(n_kv_heads), int(head_dim)
        self.c.h_ctx_len = ctypes.cast(self._ctx, ctypes.POINTER(ctypes.c_int32))
        self.c.h_q_len = ctypes.cast(self._q, ctypes.POINTER(ctypes.c_int32)) if self._q is not None else None
        self.c.softmax_scale = float(softmax_scale if softmax_scale is not None else head_dim ** -0.5)
        self.heads, self.kv_heads, self.dim = int(n_q_heads), int(n_kv_heads), int(head_dim)
        self._blocks = {}
        self._tuning = None
        self.set_tuning(attention_ctx_splits, attention_persistent, attention_grid_blocks)

    def set_tuning(self, attention_ctx_splits: int = 0, attention_persistent: int = 0, attention_grid_blocks: int = 0) -> None:
        """relaxkv_tuning of the calls made with this shape (0 = the library's automatic choice)."""
        if attention_ctx_splits or attention_persistent or attention_grid_blocks:
            self._tuning = _Tuning(int(attention_ctx_splits), int(attention_persistent), int(attention_grid_blocks))
            self.c.h_tuning = ctypes.pointer(self._tuning)
        else:
            self._tuning = None
            self.c.h_tuning = None

    @property
    def n_req(self) -> int:
        return len(self.ctx_lens)

    def context_blocks(self, block_size: int) -> int:
        """Blocks of that many tokens in all contexts (0 for a size that the library refuses)."""
        n = self._blocks.get(block_size)
        if n is None:
            n = self._blocks[block_size] = sum(-(-t // block_size) for t in self._ctx) if block_size > 0 else 0
        return n

    def ref(self):
        return ctypes.byref(self.c)


class CacheView:
    """Host-side relaxkv_cache_view over torch tensors k, v of logical shape [tokens, H_kv, D]
    (any token/head strides, D contiguous); requests start at the given token rows."""

    def __init__(self, k: torch.Tensor, v: Optional[torch.Tensor], req_token_offsets: Sequence[int]):
        assert k.dim() == 3 and k.stride(2) == 1 and k.dtype == torch.bfloat16
        if v is not None:
            assert v.shape == k.shape and v.stride() == k.stride() and v.dtype == torch.bfloat16
        self.k, self.v = k, v
        self._off = (ctypes.c_int64 * len(req_token_offsets))(*[int(x) for x in req_token_offsets])
        self.heads, self.dim = int(k.shape[1]), int(k.shape[2])
        self.room = [max(0, int(k.shape[0]) - x) for x in self._off]       # tokens behind each request's start
        self.c = _CacheView()
        self.c.k = k.data_ptr()
        self.c.v = v.data_ptr() if v is not None else None
        self.c.token_stride, self.c.head_stride = int(k.stride(0)), int(k.stride(1))
        self.c.h_req_token_offset = ctypes.cast(self._off, ctypes.POINTER(ctypes.c_int64))

    def ref(self):
        return ctypes.byref(self.c)

    def start(self, req: int) -> int:
        """Token row at which a request begins."""
        return int(self._off[req])

    def tokens(self, req: int) -> int:
        """Token rows from where a request begins to where the next one does, or to the end."""
        start = self._off[req]
        return max(0, min([int(self.k.shape[0]), *(x for x in self._off if x > start)]) - start)


class PagedStore:
    """Host-side relaxkv_paged_cache over torch tensors k, v of logical shape [n_blocks, block_size, H_kv, D] (any block, token and head
    strides, D contiguous)."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor):
        assert k.dim() == 4 and k.stride(3) == 1 and k.dtype == torch.bfloat16
        assert v.shape == k.shape and v.stride() == k.stride() and v.dtype == torch.bfloat16
        self.k, self.v, self.heads, self.dim = k, v, int(k.shape[2]), int(k.shape[3])
        self.c = _PagedCache(k.data_ptr(), v.data_ptr(), int(k.stride(0)), int(k.stride(1)), int(k.stride(2)), int(k.shape[1]), int(k.shape[0]))

    @property
    def block_size(self) -> int:
        return int(self.k.shape[1])


class QuantizedStore:
    """Host-side relaxkv_quantized_cache over torch tensors: k, v of logical shape [n_blocks, block_size, H_kv, D], int8 or float8_e4m3fn (any block,
    token and head strides, D contiguous), their exponents k_exp, v_exp int8 [n_blocks, H_kv, block_size]."""

    TYPES = {torch.int8: 0, torch.float8_e4m3fn: 1}

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_exp: torch.Tensor, v_exp: torch.Tensor):
        assert k.dim() == 4 and k.stride(3) == 1 and k.dtype in self.TYPES
        assert v.shape == k.shape and v.stride() == k.stride() and v.dtype == k.dtype
        n, block, heads, dim = (int(x) for x in k.shape)
        for e in (k_exp, v_exp):
            assert e.shape == (n, heads, block) and e.dtype == torch.int8 and e.is_contiguous()
        self.k, self.v, self.k_exp, self.v_exp, self.block_size, self.heads, self.dim = k, v, k_exp, v_exp, block, heads, dim
        self.c = _QuantizedCache(k.data_ptr(), v.data_ptr(), k_exp.data_ptr(), v_exp.data_ptr(), int(k.stride(0)), int(k.stride(1)), int(k.stride(2)),
                                 block, n, heads, self.TYPES[k.dtype])

    @classmethod
    def empty(cls, n_blocks: int, block_size: int, kv_heads: int, dim: int, dtype=torch.int8, device="cuda") -> "QuantizedStore":
        values = [torch.empty(n_blocks, block_size, kv_heads, dim, dtype=dtype, device=device) for _ in range(2)]
        return cls(*values, *(torch.empty(n_blocks, kv_heads, block_size, dtype=torch.int8, device=device) for _ in range(2)))


class Rotary:
    """Host-side relaxkv_rotary: freq float64 [rotated dims / 2] on the device."""

    SCALINGS = {"none": 0, "linear": 1, "bands": 2, "ramp": 3}

    def __init__(self, freq: torch.Tensor, interleaved: bool = False, amplitude: float = 1.0):
        assert freq.dim() == 1 and freq.dtype == torch.float64 and freq.is_contiguous()
        self.freq, self.dims, self.interleaved, self.amplitude = freq, 2 * int(freq.numel()), bool(interleaved), float(amplitude)
        self.c = _Rotary(freq.data_ptr(), self.dims, int(self.interleaved), self.amplitude)

    @classmethod
    def scaled(cls, dims: int, theta: float, scaling: str = "none", factor: float = 1.0, original_len: int = 0, low: float = 1.0, high: float = 4.0,
               interleaved: bool = False, device="cuda") -> "Rotary":
        """Frequencies theta^(-2i / dims), scaled as relaxkv_rotary_frequencies says."""
        freq, amplitude = relaxkv_rotary_frequencies(dims, theta, scaling, factor, original_len, low, high)
        return cls(torch.tensor(freq, dtype=torch.float64, device=device), interleaved, amplitude)


_INT32 = torch.int32


def _table_layout(t: torch.Tensor, n_seq: int):
    """Width and row distance of a block table of that many sequences."""
    n, width = t.shape
    if n < n_seq or t.dtype is not _INT32:
        raise ValueError(f"a block table of {n_seq} rows of int32 expected, not {n} of {t.dtype}")
    distance, one = t.stride()
    if one != 1 or (distance < width and n > 1):
        raise AssertionError("a block table's rows are contiguous and do not overlap")
    return width, max(distance, width)


class ContinuationRows:
    """Host-side relaxkv_continuation_rows: the rows of a step over sequences that continue the contexts (sequences [seq_cu[b], seq_cu[b+1])
    continue context b; at most max_rows[b] rows of it, max_len own tokens to a row).  The device tensors are those that
    relaxkv_build_block_tables writes; they are kept alive."""

    def __init__(self, seq_cu: Sequence[int], max_rows: Sequence[int], max_len: int, row_cu: torch.Tensor, row_seq: torch.Tensor,
                 row_len: Optional[torch.Tensor], block_table: Optional[torch.Tensor]):
        for t in (row_cu, row_seq, row_len, block_table):
            assert t is None or t.dtype == torch.int32
        assert len(max_rows) == len(seq_cu) - 1 and row_cu.numel() == seq_cu[-1] + 1 and row_cu.is_contiguous() and row_seq.is_contiguous()
        assert row_len is None or (row_len.is_contiguous() and row_len.numel() >= row_seq.numel())
        assert block_table is None or (block_table.shape[0] >= seq_cu[-1] and _table_layout(block_table, seq_cu[-1]))
        self._keep = (_i32(seq_cu), _i32(max_rows), row_cu, row_seq, row_len, block_table)
        self.n_req, self.n_rows = len(max_rows), row_seq.numel()
        self.c = _ContinuationRows()
        self.c.n_seq, self.c.n_rows, self.c.max_len = int(seq_cu[-1]), row_seq.numel(), int(max_len)
        if block_table is not None:
            self.c.table_width, self.c.table_stride = int(block_table.shape[1]), max(int(block_table.stride(0)), int(block_table.shape[1]))
        self.c.h_seq_cu, self.c.h_max_rows = ctypes.addressof(self._keep[0]), ctypes.addressof(self._keep[1])
        self.c.row_cu, self.c.row_seq, self.c.row_len, self.c.block_table = (_ptr(t) for t in self._keep[2:])


def relaxkv_anchor_count(ctx_len: int, ratio: float) -> int:
    return int(lib().relaxkv_anchor_count(int(ctx_len), float(ratio)))


def relaxkv_workspace_bytes(shape: Shape, n_layers: int, k: Optional[Sequence[int]] = None) -> int:
    return int(lib().relaxkv_workspace_bytes(shape.ref(), int(n_layers), _i32(k)))


def relaxkv_score_select(shape: Shape, q_layers: List[torch.Tensor], cache_layers: List[CacheView],
                         k: Sequence[int], raw_scores_out: torch.Tensor, anchors_out: Optional[torch.Tensor],
                         workspace: torch.Tensor, norm_scores_out: Optional[torch.Tensor] = None,
                         row_lse_layers: Optional[List[Optional[torch.Tensor]]] = None, stream=None) -> None:
    n_layers = len(q_layers)
    qs = (ctypes.c_void_p * n_layers)(*[q.data_ptr() for q in q_layers])
    caches = (_CacheView * n_layers)(*[c.c for c in cache_layers])
    lses = None
    if row_lse_layers is not None:
        lses = (ctypes.c_void_p * n_layers)(*[(t.data_ptr() if t is not None else None) for t in row_lse_layers])
    _check(lib().relaxkv_score_select(shape.ref(), n_layers, qs, caches, lses, _i32(k), _ptr(raw_scores_out),
                                      _ptr(norm_scores_out), _ptr(anchors_out), _ptr(workspace),
                                      workspace.nbytes, _stream(stream)),
           "relaxkv_score_select")


def relaxkv_select_topk(shape: Shape, n_layers: int, k: Sequence[int], raw_scores: torch.Tensor,
                        anchors_out: torch.Tensor, norm_scores_out: Optional[torch.Tensor] = None,
                        stream=None) -> None:
    _check(lib().relaxkv_select_topk(*_args("s.hppp.", shape.c, int(n_layers), k, raw_scores, norm_scores_out, anchors_out,
                                            _stream(stream))), "relaxkv_select_topk")


def relaxkv_build_active_sets(shape: Shape, n_layers: int, k: Sequence[int], anchors: torch.Tensor,
                              highest_layer_out: torch.Tensor, u_pos_out: torch.Tensor, u_cu_out: torch.Tensor,
                              u_rank_out: torch.Tensor, r_rank_out: torch.Tensor, r_cu_out: torch.Tensor,
                              workspace: torch.Tensor, counts_pinned: Optional[torch.Tensor] = None,
                              stream=None) -> None:
    _check(lib().relaxkv_build_active_sets(*_args("s.hppppppppp..", shape.c, int(n_layers), k, anchors, highest_layer_out, u_pos_out,
                                                  u_cu_out, u_rank_out, r_rank_out, r_cu_out, counts_pinned, workspace, workspace.nbytes,
                                                  _stream(stream))),
           "relaxkv_build_active_sets")


def relaxkv_build_active_sets_static(shape: Shape, n_layers: int, k: Sequence[int], anchors: torch.Tensor,
                                     highest_layer_out: torch.Tensor, u_pos_out: torch.Tensor,
                                     u_cu_out: torch.Tensor, u_rank_out: torch.Tensor, r_rank_out: torch.Tensor,
                                     r_cu_out: torch.Tensor, counts_pinned: Optional[torch.Tensor] = None,
                                     stream=None) -> None:
    """Same outputs as relaxkv_build_active_sets, for callers that cannot supply a workspace: the
    scratch is a fixed array inside the library (at most 8192 counts: n_req * (1 + n_layers))."""
    _check(lib().relaxkv_build_active_sets_static(*_args("s.hpppppppp.", shape.c, int(n_layers), k, anchors, highest_layer_out, u_pos_out,
                                                         u_cu_out, u_rank_out, r_rank_out, r_cu_out, counts_pinned, _stream(stream))),
           "relaxkv_build_active_sets_static")


def _attention(fn_name, shape, mode, cache, q_new, k_new, v_new, u_pos, u_cu, r_rank, r_cu_layer, max_targets,
               max_ctx, out, lse_out, workspace, stream):
    fn = getattr(lib(), fn_name)
    _check(fn(*_args("s.sppppppp.hhppp..", shape.c, int(mode), cache.c, q_new, k_new, v_new, u_pos, u_cu, r_rank, r_cu_layer,
                     q_new.shape[0], max_targets, max_ctx, out, lse_out, workspace, workspace.nbytes, _stream(stream))), fn_name)


def relaxkv_sparse_ctx_attention(shape: Shape, mode: int, cache: CacheView, q_new: torch.Tensor,
                                 k_new: Optional[torch.Tensor], v_new: Optional[torch.Tensor],
                                 u_pos: torch.Tensor, u_cu: torch.Tensor, r_rank: torch.Tensor,
                                 r_cu_layer: torch.Tensor, max_targets: Sequence[int], max_ctx: Sequence[int],
                                 out: torch.Tensor, workspace: torch.Tensor,
                                 lse_out: Optional[torch.Tensor] = None, stream=None) -> None:
    """n_target_rows is q_new.shape[0]; k_new/v_new/out must have as many rows."""
    _attention("relaxkv_sparse_ctx_attention", shape, mode, cache, q_new, k_new, v_new, u_pos, u_cu, r_rank,
               r_cu_layer, max_targets, max_ctx, out, lse_out, workspace, stream)


def relaxkv_sparse_ctx_attention_simt(shape, mode, cache, q_new, k_new, v_new, u_pos, u_cu, r_rank, r_cu_layer,
                                      max_targets, max_ctx, out, workspace, lse_out=None, stream=None) -> None:
    _attention("relaxkv_sparse_ctx_attention_simt", shape, mode, cache, q_new, k_new, v_new, u_pos, u_cu, r_rank,
               r_cu_layer, max_targets, max_ctx, out, lse_out, workspace, stream)


def relaxkv_scatter_kv(shape: Shape, cache: CacheView, k_new: torch.Tensor, v_new: torch.Tensor,
                       u_pos: torch.Tensor, u_cu: torch.Tensor, r_rank: torch.Tensor, r_cu_layer: torch.Tensor,
                       max_targets: Sequence[int], stream=None) -> None:
    _check(lib().relaxkv_scatter_kv(*_args("sspppppph.", shape.c, cache.c, k_new, v_new, u_pos, u_cu, r_rank, r_cu_layer, max_targets,
                                           _stream(stream))), "relaxkv_scatter_kv")


def relaxkv_gather_kv(shape: Shape, mode: int, cache: CacheView, k_new: Optional[torch.Tensor],
                      v_new: Optional[torch.Tensor], u_pos: torch.Tensor, u_cu: torch.Tensor, r_rank: torch.Tensor,
                      r_cu_layer: torch.Tensor, max_ctx: Sequence[int], k_ctx_out: torch.Tensor,
                      v_ctx_out: torch.Tensor, stream=None) -> None:
    _check(lib().relaxkv_gather_kv(*_args("s.spppppphpp..", shape.c, int(mode), cache.c, k_new, v_new, u_pos, u_cu, r_rank, r_cu_layer,
                                          max_ctx, k_ctx_out, v_ctx_out, k_ctx_out.shape[0], _stream(stream))), "relaxkv_gather_kv")


def relaxkv_list_attention(shape: Shape, cache: CacheView, q_new: torch.Tensor, k_new: Optional[torch.Tensor],
                           v_new: Optional[torch.Tensor], ctx_pos: torch.Tensor, ctx_cu: torch.Tensor,
                           tgt_pos: torch.Tensor, tgt_cu: torch.Tensor, max_targets: Sequence[int],
                           max_ctx: Sequence[int], out: torch.Tensor, workspace: torch.Tensor,
                           lse_out: Optional[torch.Tensor] = None, stream=None) -> None:
    _check(lib().relaxkv_list_attention(*_args("ssppppppp.hhppp..", shape.c, cache.c, q_new, k_new, v_new, ctx_pos, ctx_cu, tgt_pos, tgt_cu,
                                               q_new.shape[0], max_targets, max_ctx, out, lse_out, workspace, workspace.nbytes,
                                               _stream(stream))), "relaxkv_list_attention")


def relaxkv_cache_attention(shape: Shape, cache: CacheView, q_new: torch.Tensor, tgt_pos: torch.Tensor, tgt_cu: torch.Tensor,
                            max_targets: Sequence[int], out: torch.Tensor, workspace: torch.Tensor,
                            lse_out: Optional[torch.Tensor] = None, stream=None) -> None:
    _check(lib().relaxkv_cache_attention(*_args("ssppp.hppp..", shape.c, cache.c, q_new, tgt_pos, tgt_cu, q_new.shape[0], max_targets, out,
                                                lse_out, workspace, workspace.nbytes, _stream(stream))), "relaxkv_cache_attention")


def relaxkv_query_prefill_attention(shape: Shape, cache: CacheView, q: torch.Tensor, out: torch.Tensor, lse_out: torch.Tensor,
                                    raw_scores_out: Optional[torch.Tensor], workspace: torch.Tensor, stream=None) -> None:
    """shape.ctx_lens = context tokens, shape.q_lens = query tokens; the cache holds both (context rows first)."""
    _check(lib().relaxkv_query_prefill_attention(shape.ref(), cache.ref(), _ptr(q), _ptr(out), _ptr(lse_out),
                                                 _ptr(raw_scores_out), _ptr(workspace),
                                                 workspace.nbytes,
                                                 _stream(stream)),
           "relaxkv_query_prefill_attention")


def relaxkv_scatter_kv_lists(shape: Shape, cache: CacheView, k_new: torch.Tensor, v_new: torch.Tensor,
                             tgt_pos: torch.Tensor, tgt_cu: torch.Tensor, max_targets: Sequence[int], stream=None) -> None:
    _check(lib().relaxkv_scatter_kv_lists(*_args("sspppph.", shape.c, cache.c, k_new, v_new, tgt_pos, tgt_cu, max_targets,
                                                 _stream(stream))), "relaxkv_scatter_kv_lists")


def relaxkv_mean_scores(shape: Shape, n_layers: int, scores: torch.Tensor, mean_out: torch.Tensor, stream=None) -> None:
    _check(lib().relaxkv_mean_scores(shape.ref(), int(n_layers), _ptr(scores), _ptr(mean_out), _stream(stream)),
           "relaxkv_mean_scores")


def relaxkv_scale_scores(shape: Shape, n_layers: int, scores: torch.Tensor, factor: float, stream=None) -> None:
    """scores *= factor in place (fp32 [n_layers, sum T_c] on the device)."""
    _check(lib().relaxkv_scale_scores(shape.ref(), int(n_layers), _ptr(scores), float(factor), _stream(stream)),
           "relaxkv_scale_scores")


def relaxkv_rmsnorm(x: torch.Tensor, weight: torch.Tensor, y: torch.Tensor, eps: float, stream=None) -> None:
    _check(lib().relaxkv_rmsnorm(_ptr(x), _ptr(weight), _ptr(y), x.shape[0], int(x.shape[1]),
                                 float(eps), _stream(stream)), "relaxkv_rmsnorm")


def relaxkv_linear(x: torch.Tensor, weight: torch.Tensor, y: torch.Tensor, residual: Optional[torch.Tensor] = None,
                   stream=None) -> None:
    """y = x weight^T (+ residual); weight is [n_out, n_in]."""
    _check(lib().relaxkv_linear(_ptr(x), _ptr(weight), _ptr(residual), _ptr(y), x.shape[0],
                                int(weight.shape[0]), int(weight.shape[1]), _stream(stream)), "relaxkv_linear")


def stack_qkv(wq: torch.Tensor, wk: torch.Tensor, wv: torch.Tensor) -> torch.Tensor:
    """[Wq; Wk; Wv] along the output features: the weight layout relaxkv_linear_qkv reads (a copy, made once when the
    weights are loaded)."""
    return torch.cat([wq, wk, wv], dim=0).contiguous()


def relaxkv_linear_qkv(x: torch.Tensor, w_qkv: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, stream=None) -> None:
    """q, k, v = x Wq^T, x Wk^T, x Wv^T with w_qkv = [Wq; Wk; Wv] stacked along the output features.
    q [n, n_q] (or any contiguous view of it), k and v [n, n_kv]."""
    n = x.shape[0]
    n_q, n_kv = q.numel() // max(n, 1), k.numel() // max(n, 1)
    assert w_qkv.shape[0] == n_q + 2 * n_kv and v.numel() == k.numel()
    _check(lib().relaxkv_linear_qkv(_ptr(x), _ptr(w_qkv), _ptr(q), _ptr(k), _ptr(v), n, int(n_q), int(n_kv),
                                    int(w_qkv.shape[1]), _stream(stream)), "relaxkv_linear_qkv")


def tile_gate_up(w_gate_up: torch.Tensor) -> torch.Tensor:
    """[Wg; Wu] of shape [2 * I, K] -> the row order relaxkv_linear_swiglu reads: per block of 128 features, its gate
    rows then its up rows.  A weight-loading step (done once), not part of the path."""
    two_i, k = w_gate_up.shape
    inter = two_i // 2
    assert inter % 128 == 0
    g = w_gate_up[:inter].view(inter // 128, 128, k)
    u = w_gate_up[inter:].view(inter // 128, 128, k)
    return torch.cat([g, u], dim=1).reshape(two_i, k).contiguous()


def relaxkv_linear_swiglu(x: torch.Tensor, weight_tiled: torch.Tensor, out: torch.Tensor, stream=None) -> None:
    _check(lib().relaxkv_linear_swiglu(_ptr(x), _ptr(weight_tiled), _ptr(out), x.shape[0],
                                       int(weight_tiled.shape[0] // 2), int(weight_tiled.shape[1]), _stream(stream)),
           "relaxkv_linear_swiglu")


def relaxkv_rope(x: torch.Tensor, positions: torch.Tensor, theta: float, stream=None) -> None:
    """In place on x [rows, heads, D]; positions int32 [rows]."""
    _check(lib().relaxkv_rope(_ptr(x), x.shape[0], int(x.shape[1]), int(x.shape[2]), _ptr(positions),
                              float(theta), _stream(stream)), "relaxkv_rope")


def relaxkv_qk_norm_rope(q: torch.Tensor, k: torch.Tensor, positions: torch.Tensor, theta: float,
                         w_q_norm: Optional[torch.Tensor] = None, w_k_norm: Optional[torch.Tensor] = None, eps: float = 1e-6,
                         stream=None) -> None:
    """Per-head RMSNorm (when weights are given) and rotary embedding of q [n, H, D] and k [n, H_kv, D], in place."""
    _check(lib().relaxkv_qk_norm_rope(_ptr(q), _ptr(k), q.shape[0], int(q.shape[1]), int(k.shape[1]),
                                      int(q.shape[2]), _ptr(w_q_norm), _ptr(w_k_norm), float(eps), _ptr(positions),
                                      float(theta), _stream(stream)), "relaxkv_qk_norm_rope")


def relaxkv_qk_norm_rope_append(shape: Shape, cache: CacheView, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, tgt_pos: torch.Tensor,
                                tgt_cu: torch.Tensor, max_targets: Sequence[int], theta: float, w_q_norm: Optional[torch.Tensor] = None,
                                w_k_norm: Optional[torch.Tensor] = None, eps: float = 1e-6, stream=None) -> None:
    """relaxkv_qk_norm_rope of q [n, H, D] and k [n, H_kv, D], then relaxkv_scatter_kv_lists of k and v, both at tgt_pos."""
    _check(lib().relaxkv_qk_norm_rope_append(*_args("ssppp.pp.pph..", shape.c, cache.c, q, k, v, q.shape[0], w_q_norm, w_k_norm, float(eps),
                                                    tgt_pos, tgt_cu, max_targets, float(theta), _stream(stream))),
           "relaxkv_qk_norm_rope_append")


def relaxkv_swiglu(gate_up: torch.Tensor, out: torch.Tensor, stream=None) -> None:
    _check(lib().relaxkv_swiglu(_ptr(gate_up), _ptr(out), gate_up.shape[0], int(out.shape[1]),
                                _stream(stream)), "relaxkv_swiglu")


def relaxkv_target_positions(shape: Shape, u_pos, u_cu, r_rank, r_cu_layer, max_targets: Sequence[int],
                             positions_out: torch.Tensor, stream=None) -> None:
    _check(lib().relaxkv_target_positions(*_args("spppphp.", shape.c, u_pos, u_cu, r_rank, r_cu_layer, max_targets, positions_out,
                                                 _stream(stream))), "relaxkv_target_positions")


def relaxkv_carry_rows(shape: Shape, h_in: torch.Tensor, h_out: torch.Tensor, r_rank, r_cu_layer, r_cu_next,
                       max_next: Sequence[int], stream=None) -> None:
    _check(lib().relaxkv_carry_rows(*_args("spp.ppph.", shape.c, h_in, h_out, int(h_in.shape[1]), r_rank, r_cu_layer, r_cu_next, max_next,
                                           _stream(stream))), "relaxkv_carry_rows")


def relaxkv_continuation_workspace_bytes(shape: Shape, n_rows: int, block_size: int = 0) -> int:
    return int(lib().relaxkv_continuation_workspace_bytes(shape.ref(), int(n_rows), int(block_size)))


def relaxkv_build_block_tables(block_size: int, seq_len: torch.Tensor, new_len: torch.Tensor, seq_base: Optional[torch.Tensor],
                               free_blocks: torch.Tensor, n_free: torch.Tensor, block_table: torch.Tensor, seq_len_out: torch.Tensor,
                               n_free_out: torch.Tensor, row_cu: torch.Tensor, row_seq: torch.Tensor, row_pos: torch.Tensor,
                               row_len: torch.Tensor, row_slot: torch.Tensor, stream=None) -> None:
    """seq_len, new_len, seq_base [n_seq]; block_table [n_seq, width] (rows any distance apart); row_* [n_rows].  All int32."""
    n, n_rows, n_stack = seq_len.numel(), row_seq.numel(), free_blocks.numel()
    width, distance = _table_layout(block_table, n)
    _check(lib().relaxkv_build_block_tables(*_args("..#Iii#I.#Ip...#I#I#I#IIII.", n, int(block_size), n, seq_len, new_len, seq_base, n_stack,
                                                   free_blocks, n_stack, 1, n_free, block_table, width, distance, n_rows, n, seq_len_out,
                                                   1, n_free_out, n + 1, row_cu, n_rows, row_seq, row_pos, row_len, row_slot, _stream(stream))),
           "relaxkv_build_block_tables")


def relaxkv_qk_norm_rope_append_paged(store: PagedStore, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, positions: torch.Tensor,
                                      slots: torch.Tensor, theta: float, q_out: torch.Tensor, w_q_norm: Optional[torch.Tensor] = None,
                                      w_k_norm: Optional[torch.Tensor] = None, eps: float = 1e-6, stream=None) -> None:
    """q_out [n, H, D] = normed and rotated q (may be q); the store receives the normed and rotated k and v [n, H_kv, D] at `slots`."""
    n, heads, dim = q.shape
    kv_heads = k.shape[1]
    if kv_heads > store.heads or dim != store.dim:
        raise ValueError(f"{kv_heads} heads of {dim} for a store of {store.heads} heads of {store.dim}")
    size = n * heads * dim
    kv_size = n * kv_heads * dim
    _check(lib().relaxkv_qk_norm_rope_append_paged(*_args("s#w#ww....#WW.#II.#W.", store.c, size, q, kv_size, k, v, n, heads, kv_heads, dim, dim,
                                                          w_q_norm, w_k_norm, float(eps), n, positions, slots, float(theta), size, q_out,
                                                          _stream(stream))), "relaxkv_qk_norm_rope_append_paged")


def _fit(shape: Shape, cache: Optional[CacheView], store: Optional[PagedStore], rows: Optional[ContinuationRows]) -> None:
    """Whether a call's cache, store and rows hold what its shape says that they do."""
    if cache is not None:
        if cache.dim != shape.dim or cache.heads < shape.kv_heads:
            raise ValueError(f"a cache of {cache.heads} heads of {cache.dim} for a shape of {shape.kv_heads} heads of {shape.dim}")
        lens, room = shape.ctx_lens, cache.room
        if len(room) < len(lens) or False in map(operator.le, lens, room):
            raise ValueError(f"contexts of {lens} tokens in a cache with room for {room}")
    if store is not None and (store.dim != shape.dim or store.heads < shape.kv_heads):
        raise ValueError(f"a store of {store.heads} heads of {store.dim} for a shape of {shape.kv_heads} heads of {shape.dim}")
    if rows is not None and rows.n_req != len(shape.ctx_lens):
        raise ValueError(f"rows over {rows.n_req} contexts for a shape of {len(shape.ctx_lens)}")


def _optional(struct):
    return None if struct is None else struct.c


def _codes(before: str, cache, store, behind: str) -> str:
    """Argument codes with a cache and a store between them that may be missing."""
    return before + ("." if cache is None else "s") + ("." if store is None else "s") + behind


def relaxkv_shared_prefix_attention(shape: Shape, cache: Optional[CacheView], store: Optional[PagedStore], rows: ContinuationRows,
                                    q: torch.Tensor, out: torch.Tensor, workspace: torch.Tensor, lse_out: Optional[torch.Tensor] = None,
                                    stream=None) -> None:
    """cache: the contexts (None where all are empty); store: the sequences' own tokens (None where rows.max_len is 0)."""
    _fit(shape, cache, store, rows)
    heads = rows.n_rows * shape.heads
    _check(lib().relaxkv_shared_prefix_attention(*_args(_codes("s", cache, store, "s#ww#fp.."), shape.c, _optional(cache), _optional(store),
                                                        rows.c, heads * shape.dim, q, out, heads, lse_out, workspace, workspace.nbytes,
                                                        _stream(stream))), "relaxkv_shared_prefix_attention")


def relaxkv_block_bounds(shape: Shape, cache: Optional[CacheView], block_size: int, bounds_out: torch.Tensor, scale_out: torch.Tensor,
                         stream=None) -> None:
    """bounds_out int8 [sum of the contexts' blocks, H_kv, 2, D], scale_out fp32 [.., H_kv].  cache: None where all contexts are empty."""
    _fit(shape, cache, None, None)
    n = shape.context_blocks(block_size) * shape.kv_heads
    _check(lib().relaxkv_block_bounds(*_args(("s." if cache is None else "ss") + ".#C#F.", shape.c, _optional(cache), int(block_size),
                                             2 * shape.dim * n, bounds_out, n, scale_out, _stream(stream))), "relaxkv_block_bounds")


def relaxkv_select_blocks(shape: Shape, block_size: int, bounds: torch.Tensor, scale: torch.Tensor, rows: ContinuationRows, q: torch.Tensor,
                          n_first: int, n_last: int, blocks_out: torch.Tensor, workspace: torch.Tensor, stream=None) -> None:
    """blocks_out int32 [n_rows, H_kv, n_select]."""
    _fit(shape, None, None, rows)
    n, n_select, n_rows = shape.context_blocks(block_size) * shape.kv_heads, blocks_out.shape[2], rows.n_rows
    _check(lib().relaxkv_select_blocks(*_args("s.#c#fs#w...#ip..", shape.c, int(block_size), 2 * shape.dim * n, bounds, n, scale, rows.c,
                                              n_rows * shape.heads * shape.dim, q, n_select, int(n_first), int(n_last),
                                              n_rows * shape.kv_heads * n_select, blocks_out, workspace, workspace.nbytes, _stream(stream))),
           "relaxkv_select_blocks")


def relaxkv_block_sparse_attention(shape: Shape, cache: Optional[CacheView], store: Optional[PagedStore], rows: ContinuationRows,
                                   block_size: int, blocks: torch.Tensor, q: torch.Tensor, out: torch.Tensor, workspace: torch.Tensor,
                                   lse_out: Optional[torch.Tensor] = None, stream=None) -> None:
    """blocks int32 [n_rows, H_kv, n_select]: the context blocks that each row and KV head reads."""
    _fit(shape, cache, store, rows)
    n_select, heads = blocks.shape[2], rows.n_rows * shape.heads
    _check(lib().relaxkv_block_sparse_attention(*_args(_codes("s", cache, store, "s.#i.#ww#fp.."), shape.c, _optional(cache), _optional(store),
                                                       rows.c, int(block_size), rows.n_rows * shape.kv_heads * n_select, blocks, n_select,
                                                       heads * shape.dim, q, out, heads, lse_out, workspace, workspace.nbytes,
                                                       _stream(stream))), "relaxkv_block_sparse_attention")


def relaxkv_rotary_frequencies(dims: int, theta: float, scaling: str = "none", factor: float = 1.0, original_len: int = 0, low: float = 1.0,
                               high: float = 4.0):
    """The dims / 2 frequencies and the amplitude (scaling: a name of Rotary.SCALINGS)."""
    freq, amplitude = (ctypes.c_double * max(1, int(dims) // 2))(), ctypes.c_float()
    _check(lib().relaxkv_rotary_frequencies(int(dims), float(theta), Rotary.SCALINGS[scaling], float(factor), int(original_len), float(low), float(high),
                                            ctypes.byref(freq), ctypes.byref(amplitude)), "relaxkv_rotary_frequencies")
    return list(freq), float(amplitude.value)


def _head_rows(x: torch.Tensor, like: Optional[torch.Tensor], n: Optional[int], heads: Optional[int], dim: Optional[int]):
    """Rows, heads, dims, token and head stride of bf16 head rows [n, heads, dim] (None: any), whose heads are contiguous and which `like` (or None) is laid
    out as; ValueError for others.  The first call puts the native function in this one's place."""
    global _head_rows
    _head_rows = _native().head_rows
    return _head_rows(x, like, n, heads, dim)


def relaxkv_qk_norm_rotate(q: Optional[torch.Tensor], k: Optional[torch.Tensor], positions: torch.Tensor, rotary: Rotary, q_out: Optional[torch.Tensor] = None,
                           k_out: Optional[torch.Tensor] = None, w_q_norm: Optional[torch.Tensor] = None, w_k_norm: Optional[torch.Tensor] = None,
                           eps: float = 1e-6, stream=None) -> None:
    """Per-head RMSNorm (when weights are given) and any rotary embedding of q [n, H, D] and k [n, H_kv, D] (either may be None), into q_out and k_out, which are laid
    out like them, or in place where these are None."""
    q_out, k_out = q if q_out is None else q_out, k if k_out is None else k_out
    n = dim = None
    heads = kv_heads = q_token = q_head = k_token = k_head = 0
    if q is not None:
        n, heads, dim, q_token, q_head = _head_rows(q, q_out, None, None, None)
    if k is not None:
        n, kv_heads, dim, k_token, k_head = _head_rows(k, k_out, n, None, dim)
    if n is None:
        raise ValueError("neither q nor k")
    _check(lib().relaxkv_qk_norm_rotate(*_args("pp..pp......#WW.#Is.", q, q_out, q_token, q_head, k, k_out, k_token, k_head, n, heads, kv_heads, dim, dim,
                                               w_q_norm, w_k_norm, float(eps), n, positions, rotary.c, _stream(stream))), "relaxkv_qk_norm_rotate")


def relaxkv_append_quantized(store: QuantizedStore, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, q: Optional[torch.Tensor] = None,
                             q_out: Optional[torch.Tensor] = None, positions: Optional[torch.Tensor] = None, rotary: Optional[Rotary] = None,
                             w_q_norm: Optional[torch.Tensor] = None, w_k_norm: Optional[torch.Tensor] = None, eps: float = 1e-6, stream=None) -> None:
    """The store receives k (normed where weights are given, turned where a rotary is) and v [n, H_kv, D] at `slots`; q_out (None: q itself) = q likewise."""
    n, kv_heads, dim, k_token, k_head = _head_rows(k, v, None, store.heads, store.dim)
    heads = q_token = q_head = 0
    if q is not None:
        q_out = q if q_out is None else q_out
        _, heads, _, q_token, q_head = _head_rows(q, q_out, n, None, dim)
    elif q_out is not None:
        raise ValueError("q_out without q")
    _check(lib().relaxkv_append_quantized(*_args("spp..pp......#WW.#I" + ("." if rotary is None else "s") + "I.", store.c, q, q_out, q_token, q_head, k, v, k_token,
                                                 k_head, n, heads, kv_heads, dim, dim, w_q_norm, w_k_norm, float(eps), n, positions,
                                                 None if rotary is None else rotary.c, slots, _stream(stream))), "relaxkv_append_quantized")


def relaxkv_read_quantized(store: QuantizedStore, slots: torch.Tensor, k_out: torch.Tensor, v_out: torch.Tensor, positions: Optional[torch.Tensor] = None,
                           rotary: Optional[Rotary] = None, stream=None) -> None:
    """k_out, v_out [n, H_kv, D] = the store's rows at `slots`, the keys turned by `positions` more."""
    n, kv_heads, dim, token, head = _head_rows(k_out, v_out, None, store.heads, store.dim)
    _check(lib().relaxkv_read_quantized(*_args("s#I...I" + ("." if rotary is None else "s") + "pp...", store.c, n, slots, n, kv_heads, dim, positions,
                                               None if rotary is None else rotary.c, k_out, v_out, token, head, _stream(stream))), "relaxkv_read_quantized")


def relaxkv_quantized_workspace_bytes(n_q_heads: int, n_kv_heads: int, head_dim: int) -> int:
    return int(lib().relaxkv_quantized_workspace_bytes(int(n_q_heads), int(n_kv_heads), int(head_dim)))


def relaxkv_quantized_attention(store: QuantizedStore, rows: ContinuationRows, q: torch.Tensor, out: torch.Tensor, workspace: torch.Tensor,
                                lse_out: Optional[torch.Tensor] = None, softmax_scale: Optional[float] = None, stream=None) -> None:
    """q, out [n_rows, H, D], contiguous; softmax_scale: D^-1/2 where None."""
    n, heads, dim = q.shape
    if dim != store.dim or n != rows.n_rows:
        raise ValueError(f"{n} rows of heads of {dim} for {rows.n_rows} rows over a store of heads of {store.dim}")
    size = n * heads * dim
    _check(lib().relaxkv_quantized_attention(*_args("ss....#ww#fp..", store.c, rows.c, heads, store.heads, dim,
                                                    float(dim ** -0.5 if softmax_scale is None else softmax_scale), size, q, out, n * heads, lse_out, workspace,
                                                    workspace.nbytes, _stream(stream))), "relaxkv_quantized_attention")


def relaxkv_debug_wait_timeout(stream=None) -> None:
    """Launches the bounded-wait probe: ends after ~0.4 s with RELAXKV_ERR_TIMEOUT in the status word."""
    _check(lib().relaxkv_debug_wait_timeout(_stream(stream)), "relaxkv_debug_wait_timeout")


def relaxkv_read_device_status(stream=None):
    """Synchronises the stream; returns (status, [kernel id, block, v0, v1]) and clears the word."""
    st = ctypes.c_int32(0)
    detail = (ctypes.c_int32 * 4)()
    _check(lib().relaxkv_read_device_status(ctypes.byref(st), detail, _stream(stream)), "relaxkv_read_device_status")
    return int(st.value), list(detail)
