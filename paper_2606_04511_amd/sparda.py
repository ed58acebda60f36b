"""Thin ctypes binding of libsparda.so (argument marshalling only).

Each function keeps the C name and argument order of include/sparda.h.  Tensors are torch
tensors on the GPU (bf16 tensors as torch.bfloat16, block indices as torch.int16); they are
passed as raw pointers, and every step runs in the library's HIP kernels.  ``stream`` defaults to
torch's current stream.  A nonzero status raises SpardaError with the library's detail text.
The library must have been built (``paper_2606_04511_amd.build.build()``); there is no fallback.
"""
from __future__ import annotations

import ctypes
import os
import struct
from dataclasses import dataclass, field

import torch

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libsparda.so")

SPARDA_OK = 0
SPARDA_ERR_INVALID_ARG = -1
SPARDA_ERR_UNSUPPORTED = -2
SPARDA_ERR_WORKSPACE = -3
SPARDA_ERR_HOST_NOT_MAPPED = -4
SPARDA_ERR_HIP = -5
SPARDA_OP_FORECAST_SELECT = 1
SPARDA_OP_SPARSE_ATTN = 2
SPARDA_OP_MULTIHEAD_SELECT = 3
SPARDA_OP_INDEXER_KL = 4
SPARDA_OP_DECODE_STEP = 5
SPARDA_OP_TREE_SELECT = 6
SPARDA_OP_TREE_ATTN = 7
SPARDA_OP_PAGED_SELECT = 16
SPARDA_OP_PAGED_ATTN = 17
SPARDA_PROB_F32 = 0
SPARDA_PROB_BF16 = 1
SPARDA_F32 = 0
SPARDA_BF16 = 1
SPARDA_ROPE_HALF = 0
SPARDA_ROPE_PAIRS = 1
SPARDA_ROPE_PLAIN = 0
SPARDA_ROPE_LINEAR = 1
SPARDA_ROPE_BASE = 2
SPARDA_ROPE_BANDS = 3
SPARDA_ROPE_FACTORS = 4
SPARDA_NOALLOC_SCRATCH_BYTES = 4718592  # the static scratch of sparda_sparse_attn_noalloc (include/sparda.h)

EXPORTED = ("sparda_compress_keys", "sparda_forecast_select", "sparda_forecast_score_max", "sparda_multihead_select",
            "sparda_sparse_attn", "sparda_sparse_attn_noalloc", "sparda_gather_blocks", "sparda_stage_append_kv", "sparda_writeback_kv", "sparda_plan_staging", "sparda_indexer_kl",
            "sparda_tree_select", "sparda_tree_attn", "sparda_tree_verify", "sparda_tree_verify_workspace_size",
            "sparda_tree_commit", "sparda_rope_freqs", "sparda_rotate", "sparda_paged_append", "sparda_paged_select",
            "sparda_paged_attn", "sparda_workspace_size", "sparda_status_string", "sparda_last_error_detail")


class _CShape(ctypes.Structure):
    _fields_ = [
        ("struct_size", ctypes.c_uint32), ("batch", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
        ("group_size", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("block_size", ctypes.c_int32),
        ("cmp_kernel", ctypes.c_int32), ("cmp_stride", ctypes.c_int32), ("n_init", ctypes.c_int32),
        ("n_local", ctypes.c_int32), ("k_total", ctypes.c_int32), ("t_cap", ctypes.c_int64),
        ("nc_cap", ctypes.c_int64),
    ]


@dataclass
class SpardaShape:
    batch: int
    n_kv_heads: int
    group_size: int
    k_total: int
    t_cap: int
    nc_cap: int
    n_init: int = 1
    n_local: int = 2
    head_dim: int = 128
    block_size: int = 64
    cmp_kernel: int = 64
    cmp_stride: int = 64
    _c: _CShape = field(default=None, repr=False, compare=False)

    @property
    def n_q_heads(self) -> int:
        return self.n_kv_heads * self.group_size

    def __setattr__(self, name, value):
        object.__setattr__(self, name, value)
        object.__setattr__(self, "_c", None)  # the C struct below is of other values

    def c(self) -> _CShape:
        return _CShape(ctypes.sizeof(_CShape), self.batch, self.n_kv_heads, self.group_size, self.head_dim,
                       self.block_size, self.cmp_kernel, self.cmp_stride, self.n_init, self.n_local, self.k_total,
                       self.t_cap, self.nc_cap)

    def _struct(self) -> _CShape:
        """c() of these values, made once (0.9 us); the calls below only read it."""
        if self._c is None:
            object.__setattr__(self, "_c", self.c())
        return self._c


class _CRope(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("rot_dim", ctypes.c_int32), ("layout", ctypes.c_int32),
                ("scale", ctypes.c_float), ("freq", ctypes.c_void_p)]


class _CPages(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("page_size", ctypes.c_int32), ("n_pages", ctypes.c_int64),
                ("table_ld", ctypes.c_int64), ("page_ld", ctypes.c_int64), ("table", ctypes.c_void_p),
                ("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_cmp", ctypes.c_void_p)]


class SpardaRope:
    """A rotation (struct sparda_rope), made once for a model.  freq: float64 tensor on the GPU, radians per position."""

    def __init__(self, rot_dim: int, layout: int, freq, scale: float = 1.0):
        _expect(freq, "freq", torch.float64, rot_dim // 2)
        self.freq = freq
        self.c = _CRope(ctypes.sizeof(_CRope), rot_dim, layout, scale, _p(freq))
        self.ref = ctypes.byref(self.c)


class SpardaPages:
    """The pages of one layer (struct sparda_pages), made once: it holds the tensors and their addresses.
    table: int32 [B][pages of a sequence]; k, v: bf16 [n_pages][Hkv][P][128] (views of one pool with the same stride
    between pages are fine); k_cmp: bf16 [n_pages][Hkv][P / stride][128], dense.  What a call does not use can be None.
    The calls read the table's memory when they run: a sequence that grows, ends or moves is written into the table in place
    (one table, and so one handle per layer, for as many sequences and pages as a server has)."""

    def __init__(self, page_size: int, table, k=None, v=None, k_cmp=None):
        pools = [x for x in (k, v, k_cmp) if x is not None]
        if not pools or len({x.shape[0] for x in pools}) != 1:
            raise ValueError("k, v and k_cmp have the same number of pages")
        for x, name in ((k, "k"), (v, "v"), (k_cmp, "k_cmp")):
            if x is not None and (x.dtype != torch.bfloat16 or x.dim() != 4 or x.shape[3] != 128 or not x[0].is_contiguous()):
                raise ValueError(f"{name}: bf16 [n_pages][Hkv][tokens][128] with dense pages")
        if (k is None) != (v is None) or (k is not None and (k.stride(0) != v.stride(0) or k.shape != v.shape)):
            raise ValueError("k and v come together, with one stride between pages")
        if k is not None and k.shape[2] != page_size:
            raise ValueError(f"pages of {k.shape[2]} tokens, page_size {page_size}")
        if k_cmp is not None and not k_cmp.is_contiguous():
            raise ValueError("k_cmp is not dense")
        if table.dtype != torch.int32 or table.dim() != 2 or table.stride(1) != 1:
            raise ValueError("table: int32 [B][pages of a sequence]")
        if len({x.device for x in (table, *pools)}) != 1:
            raise ValueError("the table and the pools are on one device")
        self.page_size, self.n_seqs, self.tokens = page_size, table.shape[0], table.shape[1] * page_size
        self.kv_heads = None if k is None else k.shape[1]
        self.cmp = None if k_cmp is None else (k_cmp.shape[1], k_cmp.shape[2])
        self.tensors = (table, k, v, k_cmp)
        self.c = _CPages(ctypes.sizeof(_CPages), page_size, pools[0].shape[0],
                         table.stride(0) if table.shape[0] > 1 else table.shape[1], 0 if k is None else k.stride(0),
                         _p(table), _p(k), _p(v), _p(k_cmp))
        self.ref = ctypes.byref(self.c)

    def check(self, shape: SpardaShape):
        """The pages are those of such a shape."""
        if (self.n_seqs < shape.batch or self.tokens < shape.t_cap or self.kv_heads not in (None, shape.n_kv_heads) or
                self.cmp not in (None, (shape.n_kv_heads, self.page_size // shape.cmp_stride))):
            raise ValueError(f"pages of {self.n_seqs} sequences of {self.tokens} tokens, {self.kv_heads} KV heads, {self.cmp} "
                             f"heads and keys of a page do not go with {shape}")


class SpardaError(RuntimeError):
    def __init__(self, status: int, name: str, detail: str):
        super().__init__(f"{name} failed: {status_string(status)} ({detail})")
        self.status = status


_lib = None


def library_path() -> str:
    return _LIB_PATH


def load() -> ctypes.CDLL:
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError(f"{_LIB_PATH} is not built; run paper_2606_04511_amd.build.build() first "
                               "(there is no non-HIP fallback)")
        lib = ctypes.CDLL(_LIB_PATH)
        P, S = ctypes.c_void_p, ctypes.POINTER(_CShape)
        i32, i64 = ctypes.c_int32, ctypes.c_int64
        lib.sparda_compress_keys.argtypes = [S, P, i64, i32, i32, P, P]
        lib.sparda_forecast_select.argtypes = [S, P, i32, i64, P, P, P, P, ctypes.c_size_t, P]
        lib.sparda_forecast_score_max.argtypes = [S, P, i32, i64, P, P, P]
        lib.sparda_multihead_select.argtypes = [S, P, i32, i64, P, ctypes.c_float, P, P, P, ctypes.c_size_t, P]
        lib.sparda_sparse_attn.argtypes = [S, P, i32, i64, P, P, i32, P, P, ctypes.c_float, P, P, ctypes.c_size_t, P]
        lib.sparda_sparse_attn_noalloc.argtypes = [S, P, i32, i64, P, P, i32, P, P, ctypes.c_float, P, P]
        lib.sparda_decode_step.argtypes = [S, P, i64, P, P, P, P, ctypes.c_float, P, P, P, P, ctypes.c_size_t, P]
        lib.sparda_plan_staging.argtypes = [S, P, P, i64, P, P, P, P, P, P, P]
        lib.sparda_indexer_kl.argtypes = [S, P, P, P, P, i32, i64, ctypes.c_float, i32, P, P, P, ctypes.c_size_t, P]
        lib.sparda_gather_blocks.argtypes = [S, P, P, P, P, P, P, i32, P]
        lib.sparda_writeback_kv.argtypes = [S, P, P, i32, i64, P, P, i32, P]
        lib.sparda_stage_append_kv.argtypes = [S, P, P, i64, P, P, P, P, P]
        lib.sparda_workspace_size.argtypes = [S, i32, i32, i64, ctypes.POINTER(ctypes.c_size_t)]
        sz = ctypes.c_size_t
        lib.sparda_tree_select.argtypes = [S, P, i32, P, i64, P, P, P, P, P, sz, P]
        lib.sparda_tree_attn.argtypes = [S, P, i32, P, i64, P, P, P, P, P, i32, P, P, ctypes.c_float, P, P, sz, P]
        lib.sparda_tree_verify.argtypes = [S, i32, i32, i64, i32, P, P, P, P, P, P, P, P, P, sz, P]
        lib.sparda_tree_verify_workspace_size.argtypes = [S, i32, i32, ctypes.POINTER(sz)]
        lib.sparda_tree_commit.argtypes = [S, i32, P, P, P, i32, P, P, P, P, P, P, P]
        R, W, G = ctypes.POINTER(_CRope), ctypes.c_char_p, ctypes.POINTER(_CPages)  # W: packed bytes (_rows)
        f64 = ctypes.c_double
        lib.sparda_rope_freqs.argtypes = [i32, f64, i32, f64, f64, f64, f64, P, P, ctypes.POINTER(ctypes.c_float)]
        lib.sparda_rotate.argtypes = [R, i32, i32, i32, i64, W, P, i64, W, i32, P]
        lib.sparda_paged_append.argtypes = [S, G, R, i32, P, P, W, W, W, W, W, W, P, P]
        lib.sparda_paged_select.argtypes = [S, G, P, P, i64, P, P, P, sz, P]
        lib.sparda_paged_attn.argtypes = [S, G, P, P, i64, P, P, ctypes.c_float, P, P, sz, P]
        for name in ("sparda_rope_freqs", "sparda_rotate", "sparda_paged_append", "sparda_paged_select",
                     "sparda_paged_attn", "sparda_tree_select", "sparda_tree_attn", "sparda_tree_verify",
                     "sparda_tree_verify_workspace_size", "sparda_tree_commit",
                     "sparda_compress_keys", "sparda_forecast_select", "sparda_forecast_score_max",
                     "sparda_multihead_select", "sparda_sparse_attn", "sparda_sparse_attn_noalloc", "sparda_decode_step",
                     "sparda_gather_blocks",
                     "sparda_stage_append_kv", "sparda_writeback_kv", "sparda_plan_staging", "sparda_indexer_kl",
                     "sparda_workspace_size"):
            getattr(lib, name).restype = ctypes.c_int
        lib.sparda_status_string.argtypes = [ctypes.c_int]
        lib.sparda_status_string.restype = ctypes.c_char_p
        lib.sparda_last_error_detail.argtypes = []
        lib.sparda_last_error_detail.restype = ctypes.c_char_p
        _lib = lib
    return _lib


def status_string(status: int) -> str:
    return load().sparda_status_string(int(status)).decode()


def last_error_detail() -> str:
    return load().sparda_last_error_detail().decode()


def _check(rc: int, name: str):
    if rc != SPARDA_OK:
        raise SpardaError(rc, name, last_error_detail())


def _p(x):
    """Raw pointer of a tensor (or an int address / None)."""
    if x is None:
        return None
    if isinstance(x, int):
        return x
    return x.data_ptr()


def _expect(x, name: str, dtype, numel: int):
    """A dense tensor of `numel` elements at least (ints and None pass: raw addresses)."""
    if x is None or isinstance(x, int):
        return
    if x.dtype != dtype or not x.is_contiguous() or x.numel() < numel:
        raise ValueError(f"{name}: {numel} dense elements of {dtype} expected")


def _present() -> int:
    """The current device, whose stream the calls go to (-2: none in use; a tensor in host memory is on -1)."""
    return _device() if torch.cuda.is_initialized() else -2


def _elsewhere(x, dev: int):
    raise ValueError(f"a tensor is on {x.device}, the current device is {'cuda:%d' % dev if dev >= 0 else 'not in use'}")


def _here(dev: int, *tensors):
    """The tensors are in the memory of device `dev`."""
    for x in tensors:
        if x is not None and not isinstance(x, (int, tuple)) and x.get_device() != dev:
            _elsewhere(x, dev)


def _dense(x, name: str, dtype, numel: int, dev: int):
    """The address of a dense tensor of `numel` elements at least on device `dev` (ints and None pass: raw addresses)."""
    if x is None or isinstance(x, int):
        return x
    if x.dtype is not dtype or x.numel() < numel or not x.is_contiguous():
        raise ValueError(f"{name}: {numel} dense elements of {dtype} expected")
    if x.get_device() != dev:
        _elsewhere(x, dev)
    return x.data_ptr()


def _expect_pos(pos, batch: int, n_tok: int, pos_ld: int):
    """Positions [b pos_ld + t], b < batch, t < n_tok, lie in the tensor: a dense one of as many elements, or rows pos_ld apart."""
    if pos is None or isinstance(pos, int) or batch <= 0 or n_tok <= 0:
        return
    if pos.dtype != torch.int32 or not (
            pos.numel() >= (batch - 1) * pos_ld + n_tok if pos.is_contiguous() else
            pos.dim() == 2 and pos.shape[0] >= (batch if pos_ld else 1) and pos.shape[1] >= n_tok and
            (n_tok == 1 or pos.stride(1) == 1) and (batch == 1 or pos_ld == 0 or pos.stride(0) == pos_ld)):
        raise ValueError(f"pos: int32, {n_tok} dense positions of {batch} sequences {pos_ld} apart expected")


def _space(ws, ws_bytes: int, dev: int):
    """Address and bytes of a workspace (0: all of the tensor)."""
    if ws is None or isinstance(ws, int):
        return ws, ws_bytes
    n = ws.nbytes
    if ws_bytes > n or not ws.is_contiguous():
        raise ValueError(f"ws: a dense tensor of {ws_bytes or n} bytes expected")
    if ws.get_device() != dev:
        _elsewhere(ws, dev)
    return ws.data_ptr(), ws_bytes or n


_pack_rows = struct.Struct("=Qqqq").pack  # struct sparda_rows


def _rows(x, name: str, shape, dtype):
    """struct sparda_rows of a tensor [B][heads][tokens][128] of any strides, or of (address, ld_batch, ld_head, ld_token).
    Packed bytes: a ctypes structure costs 1.7 us, and an append has six."""
    if x is None:
        return None
    if isinstance(x, tuple):
        return _pack_rows(x[0] or 0, *x[1:])
    b, h, t, d = x.stride()  # (ValueError where there are not four)
    if d != 1 or x.shape != shape or x.dtype != dtype:
        raise ValueError(f"{name}: {tuple(shape)} of {dtype} expected, its last dimension dense")
    return _pack_rows(x.data_ptr(), b, h, t)


_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
# The current stream's handle without a Stream object around it (0.4 us instead of 2.9 us per call).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream, dev: int = -1):
    """A stream's handle; None: the current one, of device `dev` where the caller has asked for that already."""
    if stream is None:
        if dev >= 0 and _raw_stream is not None:
            return _raw_stream(dev)
        if _raw_stream is not None and torch.cuda.is_initialized():
            return _raw_stream(_device())
        return torch.cuda.current_stream().cuda_stream if torch.cuda.is_available() else 0
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def sparda_workspace_size(shape: SpardaShape, op: int, n_q: int, q_pos0: int) -> int:
    n = ctypes.c_size_t(0)
    cs = shape._struct()
    _check(load().sparda_workspace_size(ctypes.byref(cs), op, n_q, q_pos0, ctypes.byref(n)), "sparda_workspace_size")
    return int(n.value)


def sparda_compress_keys(shape: SpardaShape, k_cache, t_ctx: int, win_begin: int, win_end: int, k_cmp, stream=None):
    cs = shape._struct()
    _check(load().sparda_compress_keys(ctypes.byref(cs), _p(k_cache), t_ctx, win_begin, win_end, _p(k_cmp),
                                       _stream(stream)), "sparda_compress_keys")


def sparda_forecast_select(shape: SpardaShape, f, n_q: int, q_pos0: int, k_cmp, sel, cnt, ws=None, ws_bytes: int = 0,
                           stream=None):
    cs = shape._struct()
    if ws is not None and not isinstance(ws, int) and ws_bytes == 0:
        ws_bytes = ws.numel() * ws.element_size()
    _check(load().sparda_forecast_select(ctypes.byref(cs), _p(f), n_q, q_pos0, _p(k_cmp), _p(sel), _p(cnt), _p(ws),
                                         ws_bytes, _stream(stream)), "sparda_forecast_select")


def sparda_forecast_score_max(shape: SpardaShape, f, n_q: int, q_pos0: int, k_cmp, row_max, stream=None):
    cs = shape._struct()
    _check(load().sparda_forecast_score_max(ctypes.byref(cs), _p(f), n_q, q_pos0, _p(k_cmp), _p(row_max),
                                            _stream(stream)), "sparda_forecast_score_max")


def sparda_multihead_select(shape: SpardaShape, q, n_q: int, q_pos0: int, k_cmp, sm_scale: float, sel, cnt, ws=None,
                            ws_bytes: int = 0, stream=None):
    cs = shape._struct()
    if ws is not None and not isinstance(ws, int) and ws_bytes == 0:
        ws_bytes = ws.numel() * ws.element_size()
    _check(load().sparda_multihead_select(ctypes.byref(cs), _p(q), n_q, q_pos0, _p(k_cmp), float(sm_scale), _p(sel),
                                          _p(cnt), _p(ws), ws_bytes, _stream(stream)), "sparda_multihead_select")


def sparda_sparse_attn(shape: SpardaShape, q, n_q: int, q_pos0: int, k, v, kv_mode: int, sel, cnt, sm_scale: float, o,
                       ws=None, ws_bytes: int = 0, stream=None):
    cs = shape._struct()
    if ws is not None and not isinstance(ws, int) and ws_bytes == 0:
        ws_bytes = ws.numel() * ws.element_size()
    _check(load().sparda_sparse_attn(ctypes.byref(cs), _p(q), n_q, q_pos0, _p(k), _p(v), kv_mode, _p(sel), _p(cnt),
                                     float(sm_scale), _p(o), _p(ws), ws_bytes, _stream(stream)), "sparda_sparse_attn")


def sparda_decode_step(shape: SpardaShape, f, q_pos: int, k_cmp, q, k, v, sm_scale: float, sel, cnt, o, ws=None,
                       ws_bytes: int = 0, stream=None):
    cs = shape._struct()
    if ws is not None and not isinstance(ws, int) and ws_bytes == 0:
        ws_bytes = ws.numel() * ws.element_size()
    _check(load().sparda_decode_step(ctypes.byref(cs), _p(f), q_pos, _p(k_cmp), _p(q), _p(k), _p(v), float(sm_scale),
                                     _p(sel), _p(cnt), _p(o), _p(ws), ws_bytes, _stream(stream)), "sparda_decode_step")


def sparda_sparse_attn_noalloc(shape: SpardaShape, q, n_q: int, q_pos0: int, k, v, kv_mode: int, sel, cnt,
                               sm_scale: float, o, stream=None):
    cs = shape._struct()
    _check(load().sparda_sparse_attn_noalloc(ctypes.byref(cs), _p(q), n_q, q_pos0, _p(k), _p(v), kv_mode, _p(sel),
                                             _p(cnt), float(sm_scale), _p(o), _stream(stream)),
           "sparda_sparse_attn_noalloc")


def sparda_gather_blocks(shape: SpardaShape, host_k, host_v, sel, cnt, stage_k, stage_v, n_workgroups: int,
                         stream=None):
    cs = shape._struct()
    _check(load().sparda_gather_blocks(ctypes.byref(cs), _p(host_k), _p(host_v), _p(sel), _p(cnt), _p(stage_k),
                                       _p(stage_v), n_workgroups, _stream(stream)), "sparda_gather_blocks")


def sparda_stage_append_kv(shape: SpardaShape, k_new, v_new, q_pos: int, sel, cnt, stage_k, stage_v, stream=None):
    cs = shape._struct()
    _check(load().sparda_stage_append_kv(ctypes.byref(cs), _p(k_new), _p(v_new), q_pos, _p(sel), _p(cnt), _p(stage_k),
                                         _p(stage_v), _stream(stream)), "sparda_stage_append_kv")


def sparda_writeback_kv(shape: SpardaShape, k_new, v_new, n_new: int, pos0: int, host_k, host_v, n_workgroups: int,
                        stream=None):
    cs = shape._struct()
    _check(load().sparda_writeback_kv(ctypes.byref(cs), _p(k_new), _p(v_new), n_new, pos0, _p(host_k), _p(host_v),
                                      n_workgroups, _stream(stream)), "sparda_writeback_kv")


def sparda_plan_staging(shape: SpardaShape, sel, cnt, q_pos: int, slot_blk, slot_len, fetch, sel_staged, stage_cnt,
                        n_fetch, stream=None):
    cs = shape._struct()
    _check(load().sparda_plan_staging(ctypes.byref(cs), _p(sel), _p(cnt), q_pos, _p(slot_blk), _p(slot_len), _p(fetch),
                                      _p(sel_staged), _p(stage_cnt), _p(n_fetch), _stream(stream)),
           "sparda_plan_staging")


def sparda_indexer_kl(shape: SpardaShape, q, k, f, k_cmp, n_q: int, q_pos0: int, sm_scale: float, k_top: int, loss, d_f,
                      ws=None, ws_bytes: int = 0, stream=None):
    cs = shape._struct()
    if ws is not None and not isinstance(ws, int) and ws_bytes == 0:
        ws_bytes = ws.numel() * ws.element_size()
    _check(load().sparda_indexer_kl(ctypes.byref(cs), _p(q), _p(k), _p(f), _p(k_cmp), n_q, q_pos0, float(sm_scale),
                                    k_top, _p(loss), _p(d_f), _p(ws), ws_bytes, _stream(stream)), "sparda_indexer_kl")


def sparda_tree_select(shape: SpardaShape, f, n_nodes: int, t_ctx, t_max: int, parent, k_cmp, sel, cnt, ws=None,
                       ws_bytes: int = 0, stream=None):
    cs = shape._struct()
    if ws is not None and not isinstance(ws, int) and ws_bytes == 0:
        ws_bytes = ws.numel() * ws.element_size()
    _check(load().sparda_tree_select(ctypes.byref(cs), _p(f), n_nodes, _p(t_ctx), t_max, _p(parent), _p(k_cmp), _p(sel),
                                     _p(cnt), _p(ws), ws_bytes, _stream(stream)), "sparda_tree_select")


def sparda_tree_attn(shape: SpardaShape, q, n_nodes: int, t_ctx, t_max: int, parent, k, v, k_tree, v_tree, n_sel: int,
                     sel, cnt, sm_scale: float, o, ws=None, ws_bytes: int = 0, stream=None):
    cs = shape._struct()
    if ws is not None and not isinstance(ws, int) and ws_bytes == 0:
        ws_bytes = ws.numel() * ws.element_size()
    _check(load().sparda_tree_attn(ctypes.byref(cs), _p(q), n_nodes, _p(t_ctx), t_max, _p(parent), _p(k), _p(v),
                                   _p(k_tree), _p(v_tree), n_sel, _p(sel), _p(cnt), float(sm_scale), _p(o), _p(ws),
                                   ws_bytes, _stream(stream)), "sparda_tree_attn")


def sparda_tree_verify_workspace_size(shape: SpardaShape, n_nodes: int, vocab: int) -> int:
    n = ctypes.c_size_t(0)
    cs = shape._struct()
    _check(load().sparda_tree_verify_workspace_size(ctypes.byref(cs), n_nodes, vocab, ctypes.byref(n)),
           "sparda_tree_verify_workspace_size")
    return int(n.value)


def sparda_tree_verify(shape: SpardaShape, n_nodes: int, vocab: int, ld: int, prob_type: int, p, q, tokens, parent, u,
                       path, n_path, next_token, ws=None, ws_bytes: int = 0, stream=None):
    cs = shape._struct()
    if ws is not None and not isinstance(ws, int) and ws_bytes == 0:
        ws_bytes = ws.numel() * ws.element_size()
    _check(load().sparda_tree_verify(ctypes.byref(cs), n_nodes, vocab, ld, prob_type, _p(p), _p(q), _p(tokens),
                                     _p(parent), _p(u), _p(path), _p(n_path), _p(next_token), _p(ws), ws_bytes,
                                     _stream(stream)), "sparda_tree_verify")


def layer_pointers(tensors):
    """The table of one pointer per layer that sparda_tree_commit takes.  It holds addresses: the tensors must stay
    alive, and a table can be kept as long as they do."""
    return (ctypes.c_void_p * len(tensors))(*[_p(x) for x in tensors])


def _table(x, n_layers: int):
    """A layer table: one made by layer_pointers, or a sequence of tensors."""
    if x is None:
        return None
    if len(x) != n_layers:
        raise ValueError(f"{len(x)} layers in a table of {n_layers}")
    return x if isinstance(x, ctypes.Array) else layer_pointers(x)


def sparda_tree_commit(shape: SpardaShape, n_nodes: int, t_ctx, path, n_path, n_layers: int, k_tree, v_tree, k_cache,
                       v_cache, k_cmp, t_new, stream=None):
    cs = shape._struct()
    _check(load().sparda_tree_commit(ctypes.byref(cs), n_nodes, _p(t_ctx), _p(path), _p(n_path), n_layers,
                                     _table(k_tree, n_layers), _table(v_tree, n_layers), _table(k_cache, n_layers),
                                     _table(v_cache, n_layers), _table(k_cmp, n_layers), _p(t_new), _stream(stream)),
           "sparda_tree_commit")


def sparda_rope_freqs(rot_dim: int, base: float, scaling: int = SPARDA_ROPE_PLAIN, factor: float = 1.0, t_train: float = 0.0,
                      low: float = 1.0, high: float = 32.0, factors=None):
    """(float64 CPU tensor [rot_dim / 2] of radians per position, scale)."""
    freq = torch.empty(max(rot_dim // 2, 1), dtype=torch.float64)
    scale = ctypes.c_float(0.0)
    if factors is not None:
        factors = torch.as_tensor(factors, dtype=torch.float64, device="cpu").contiguous()
        _expect(factors, "factors", torch.float64, rot_dim // 2)
    _check(load().sparda_rope_freqs(rot_dim, base, scaling, factor, t_train, low, high, _p(factors), _p(freq),
                                    ctypes.byref(scale)), "sparda_rope_freqs")
    return freq, float(scale.value)


def sparda_rotate(rope: SpardaRope, type: int, batch: int, n_heads: int, n_tok: int, x, pos, pos_ld: int, y,
                  backward: bool = False, stream=None):
    dtype, size = torch.float32 if type == SPARDA_F32 else torch.bfloat16, (batch, n_heads, n_tok, 128)
    dev = _present()
    _expect_pos(pos, batch, n_tok, pos_ld)
    _here(dev, rope.freq, x, y, pos)
    _check(load().sparda_rotate(rope.ref, type, batch, n_heads, n_tok, _rows(x, "x", size, dtype), _p(pos),
                                pos_ld, _rows(y, "y", size, dtype), int(backward), _stream(stream, dev)), "sparda_rotate")


def sparda_paged_append(shape: SpardaShape, pages: SpardaPages, rope, n_max: int, n_new, t_ctx, k_new, v_new, q, q_out, f,
                        f_out, t_new, stream=None):
    cs, b, h, bf, dev = shape._struct(), shape.batch, shape.n_kv_heads, torch.bfloat16, _present()
    kv, hq, i32 = (b, h, n_max, 128), (b, h * shape.group_size, n_max, 128), torch.int32
    pages.check(shape)
    n_new, t_ctx, t_new = (_dense(n_new, "n_new", i32, b, dev), _dense(t_ctx, "t_ctx", i32, b, dev),
                           _dense(t_new, "t_new", i32, b, dev))
    _here(dev, rope.freq if rope else None, pages.tensors[0], k_new, v_new, q, q_out, f, f_out)
    _check(load().sparda_paged_append(ctypes.byref(cs), pages.ref, rope.ref if rope else None, n_max,
                                      n_new, t_ctx, _rows(k_new, "k_new", kv, bf), _rows(v_new, "v_new", kv, bf),
                                      _rows(q, "q", hq, bf), _rows(q_out, "q_out", hq, bf), _rows(f, "f", kv, bf),
                                      _rows(f_out, "f_out", kv, bf), t_new, _stream(stream, dev)), "sparda_paged_append")


def sparda_paged_select(shape: SpardaShape, pages: SpardaPages, f, t_ctx, t_max: int, sel, cnt, ws=None, ws_bytes: int = 0,
                        stream=None):
    cs, b, rows, dev = shape._struct(), shape.batch, shape.batch * shape.n_kv_heads, _present()
    pages.check(shape)
    _here(dev, pages.tensors[0])
    space, size = _space(ws, ws_bytes, dev)
    _check(load().sparda_paged_select(ctypes.byref(cs), pages.ref, _dense(f, "f", torch.bfloat16, rows * 128, dev),
                                      _dense(t_ctx, "t_ctx", torch.int32, b, dev), t_max,
                                      _dense(sel, "sel", torch.int16, rows * shape.k_total, dev),
                                      _dense(cnt, "cnt", torch.int16, rows, dev), space, size, _stream(stream, dev)),
           "sparda_paged_select")


def sparda_paged_attn(shape: SpardaShape, pages: SpardaPages, q, t_ctx, t_max: int, sel, cnt, sm_scale: float, o, ws=None,
                      ws_bytes: int = 0, stream=None):
    cs, b, rows, dev = shape._struct(), shape.batch, shape.batch * shape.n_kv_heads, _present()
    size = rows * shape.group_size * 128
    pages.check(shape)
    _here(dev, pages.tensors[0])
    space, ws_bytes = _space(ws, ws_bytes, dev)
    _check(load().sparda_paged_attn(ctypes.byref(cs), pages.ref, _dense(q, "q", torch.bfloat16, size, dev),
                                    _dense(t_ctx, "t_ctx", torch.int32, b, dev), t_max,
                                    _dense(sel, "sel", torch.int16, rows * shape.k_total, dev),
                                    _dense(cnt, "cnt", torch.int16, rows, dev), float(sm_scale),
                                    _dense(o, "o", torch.bfloat16, size, dev), space, ws_bytes, _stream(stream, dev)),
           "sparda_paged_attn")
