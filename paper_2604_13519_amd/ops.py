"""Binding of the device-tensor operators of libtoolspec_hip.so (include/toolspec_ops.h) for torch tensors.

Function names mirror the header.  A call checks what the tensors themselves tell (types, shapes, devices, contiguity
within a row), allocates outputs that it is not given, and enqueues on the current stream of the tensors' GPU; whatever
is wrong raises before anything is enqueued.  The arithmetic is the library's: there is no fallback.  No call has a
backward pass: while gradients are recorded, a tensor that requires one is refused.

Import this module (or torch) before the library is loaded: it then runs on torch's HIP runtime, and not on one of its own.
"""
import ctypes as C
import struct

import numpy as np
import torch

from . import binding
from .binding import TS_DTYPE_BF16, TS_DTYPE_F32, TS_PAGE_SIZE

EXPORTS = ("ts_mx_quantize", "ts_mx_dequantize", "ts_mx_packed_bytes", "ts_mx_pack", "ts_mx_project", "ts_kv_layer_pages", "ts_kv_page_table",
           "ts_kv_extend", "ts_kv_append", "ts_kv_attend", "ts_kv_attend_workspace", "ts_kv_append_norm_rope", "ts_kv_read", "ts_kv_attend_rows",
           "ts_kv_attend_rows_workspace")

TS_DTYPE_E4M3 = 3                                          # pages of 8-bit values
_DTYPES = {torch.float32: TS_DTYPE_F32, torch.bfloat16: TS_DTYPE_BF16}
_RECORD = 16 * 4 * 17                                      # bytes of packed weights per 16 rows and 128 columns


class ts_kv_pages(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("n_pages", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("dtype", C.c_int32)]


class ts_kv_append_args(C.Structure):
    _fields_ = [("pages", ts_kv_pages), ("table", C.c_void_p), ("table_stride", C.c_int64), ("table_width", C.c_int32),
                ("lengths", C.c_void_p), ("row_offsets", C.c_void_p),
                ("n_seqs", C.c_int32), ("n_rows", C.c_int32), ("n_q_heads", C.c_int32), ("dtype", C.c_int32),
                ("q", C.c_void_p), ("q_stride", C.c_int64), ("k", C.c_void_p), ("k_stride", C.c_int64), ("v", C.c_void_p), ("v_stride", C.c_int64),
                ("q_out", C.c_void_p), ("q_out_stride", C.c_int64), ("rope_theta", C.c_float)]


class ts_kv_attend_args(C.Structure):
    _fields_ = [("pages", ts_kv_pages), ("table", C.c_void_p), ("table_stride", C.c_int64), ("table_width", C.c_int32), ("lengths", C.c_void_p),
                ("n_seqs", C.c_int32), ("max_len", C.c_int32), ("window", C.c_int32), ("n_q_heads", C.c_int32), ("dtype", C.c_int32),
                ("q", C.c_void_p), ("q_stride", C.c_int64), ("out", C.c_void_p), ("out_stride", C.c_int64), ("lse", C.c_void_p), ("scale", C.c_float),
                ("workspace", C.c_void_p), ("workspace_bytes", C.c_uint64)]


class ts_kv_pages_any(C.Structure):
    _fields_ = [("pages", ts_kv_pages), ("k_scales", C.c_void_p), ("v_scales", C.c_void_p)]


class ts_kv_append_norm_rope_args(C.Structure):
    _fields_ = [("cache", ts_kv_pages_any), ("table", C.c_void_p), ("table_stride", C.c_int64), ("table_width", C.c_int32),
                ("lengths", C.c_void_p), ("row_offsets", C.c_void_p), ("positions", C.c_void_p),
                ("n_seqs", C.c_int32), ("n_rows", C.c_int32), ("n_q_heads", C.c_int32), ("dtype", C.c_int32),
                ("q", C.c_void_p), ("q_stride", C.c_int64), ("k", C.c_void_p), ("k_stride", C.c_int64), ("v", C.c_void_p), ("v_stride", C.c_int64),
                ("q_out", C.c_void_p), ("q_out_stride", C.c_int64), ("q_norm", C.c_void_p), ("k_norm", C.c_void_p),
                ("norm_dtype", C.c_int32), ("norm_eps", C.c_float), ("rope_freqs", C.c_void_p), ("rope_theta", C.c_float), ("rope_magnitude", C.c_float),
                ("rope_dim", C.c_int32), ("rope_pairs", C.c_int32)]


class ts_kv_read_args(C.Structure):
    _fields_ = [("cache", ts_kv_pages_any), ("table", C.c_void_p), ("table_stride", C.c_int64), ("table_width", C.c_int32),
                ("starts", C.c_void_p), ("row_offsets", C.c_void_p), ("n_seqs", C.c_int32), ("n_rows", C.c_int32), ("dtype", C.c_int32), ("zero_rest", C.c_int32),
                ("k_out", C.c_void_p), ("k_stride", C.c_int64), ("v_out", C.c_void_p), ("v_stride", C.c_int64)]


class ts_kv_attend_rows_args(C.Structure):
    _fields_ = [("cache", ts_kv_pages_any), ("table", C.c_void_p), ("table_stride", C.c_int64), ("table_width", C.c_int32),
                ("lengths", C.c_void_p), ("row_offsets", C.c_void_p), ("ancestors", C.c_void_p),
                ("n_seqs", C.c_int32), ("n_rows", C.c_int32), ("max_len", C.c_int32), ("window", C.c_int32), ("n_q_heads", C.c_int32), ("dtype", C.c_int32),
                ("q", C.c_void_p), ("q_stride", C.c_int64), ("out", C.c_void_p), ("out_stride", C.c_int64), ("lse", C.c_void_p), ("scale", C.c_float),
                ("workspace", C.c_void_p), ("workspace_bytes", C.c_uint64)]


def _packer(cls):
    """Packs the members of a structure, those of its own structures in place: a quarter of the time that building the structure takes."""
    def codes(c):
        return "".join({C.c_void_p: "P", C.c_int32: "i", C.c_int64: "q", C.c_uint64: "Q", C.c_float: "f"}.get(t) or codes(t) for _, t in c._fields_)
    fmt = "@" + codes(cls)
    fmt += "%dx" % (C.sizeof(cls) - struct.calcsize(fmt))  # to the end of the structure
    return struct.Struct(fmt).pack


_pack_append, _pack_attend = _packer(ts_kv_append_args), _packer(ts_kv_attend_args)
_pack_append_norm_rope, _pack_read, _pack_rows = _packer(ts_kv_append_norm_rope_args), _packer(ts_kv_read_args), _packer(ts_kv_attend_rows_args)
_lib = None


def _load():
    global _lib
    lib = binding.load_library()
    if _lib is None:
        with open("/proc/self/maps") as maps:
            runtimes = {line.split()[-1] for line in maps if "libamdhip64" in line}
        if len(runtimes) > 1:                              # torch's and the system's: neither knows the other's memory and streams
            raise RuntimeError("the library was loaded before torch, and each uses a HIP runtime of its own (%s): import torch, or this module, before "
                               "binding.load_library" % ", ".join(sorted(runtimes)))
        p, i32, i64 = C.c_void_p, C.c_int32, C.c_int64
        for name, args in {
            "ts_mx_quantize": [p, i32, i64, i64, i64, p, p, p],
            "ts_mx_dequantize": [p, p, i64, i64, p, i32, i64, p],
            "ts_mx_packed_bytes": [i32, i32, C.POINTER(C.c_uint64)],
            "ts_mx_pack": [p, p, i32, i32, p, p],
            "ts_mx_project": [p, i32, i32, p, i32, i64, i64, p, i64, p],
            "ts_kv_layer_pages": [p, i32, C.POINTER(ts_kv_pages)],
            "ts_kv_page_table": [p, C.POINTER(i32), i32],
            "ts_kv_extend": [p, i32, p],
            "ts_kv_append": [p, p],
            "ts_kv_attend": [p, p],
            "ts_kv_attend_workspace": [i32, i32, i32, i32, i32, i32, C.POINTER(C.c_uint64)],
            "ts_kv_append_norm_rope": [p, p],
            "ts_kv_read": [p, p],
            "ts_kv_attend_rows": [p, p],
            "ts_kv_attend_rows_workspace": [i32, i32, i32, i32, i32, i32, i32, C.POINTER(C.c_uint64)],
        }.items():
            fn = getattr(lib, name)
            fn.argtypes, fn.restype = args, i32
        _lib = lib
    return lib


_stream_of = torch._C._cuda_getCurrentRawStream           # the current stream's handle without a Python object around it


def _stream(t):
    return _stream_of(t.get_device())


def _refuse(what, *args):
    raise ValueError(what % args)


def _no_gradient(name):
    if torch.is_grad_enabled():
        _refuse("%s requires a gradient, and these calls have none: detach it, or call them under torch.no_grad()", name)


def _int(v, name):
    """An int32 argument: ctypes would cut a larger one to its low bits."""
    if not -(1 << 31) <= v < 1 << 31:
        _refuse("%s: %d does not fit 32 bits", name, v)
    return v


def _out_of_range(e):
    raise ValueError("an argument is out of range: %s" % e) from None


def _rows(t, name, cols=None, dtype=None):
    """A matrix whose rows are contiguous; the distance between rows is free.  (address, distance)"""
    shape = t.shape
    if len(shape) != 2:
        _refuse("%s: a matrix with contiguous rows is needed, got shape %s", name, tuple(shape))
    n, width = shape
    dist, step = t.stride()
    if step != 1 or dist < width:                          # one column, one row: any distance will do
        if (step != 1 and width > 1) or (dist < width and n > 1):
            _refuse("%s: a matrix with contiguous rows is needed, got shape %s, strides %s", name, tuple(shape), t.stride())
        dist = max(dist, width)
    if cols is not None and width != cols:
        _refuse("%s: rows of %d values are needed, got %d", name, cols, width)
    has = t.dtype
    if has is not dtype and (dtype is not None or has not in _DTYPES):
        raise TypeError("%s: %s is needed, got %s" % (name, dtype or "float32 or bfloat16", has))
    if t.requires_grad:
        _no_gradient(name)
    if not t.is_cuda:
        _refuse("%s is not on a GPU", name)
    return t.data_ptr(), dist


def _ints(t, name, n):
    if t.dtype is not torch.int32 or not t.is_cuda or t.dim() != 1 or not t.is_contiguous() or t.shape[0] < n:
        _refuse("%s: at least %s contiguous int32 on a GPU are needed, got %s %s", name, n, t.dtype, tuple(t.shape))
    return t.data_ptr()


def _bytes(t, name, shape=None):
    if t.dtype is not torch.uint8 or not t.is_cuda or not t.is_contiguous() or (shape is not None and t.shape != shape):
        _refuse("%s: a contiguous uint8 tensor%s on a GPU is needed, got %s %s", name, " of shape %s" % (shape,) if shape else "", t.dtype, tuple(t.shape))
    return t.data_ptr()


# ---- 4-bit microscaled values ------------------------------------------------------------
def ts_mx_quantize(x, codes=None, scales=None):
    """x [rows][cols] fp32 or bf16 -> (codes uint8 [rows][16 * blocks], scales uint8 [rows][blocks]), blocks = ceil(cols / 32)."""
    lib = _lib or _load()
    px, stride = _rows(x, "x")
    rows, cols = x.shape
    blocks = (cols + 31) // 32
    if codes is None:
        codes = x.new_empty((rows, 16 * blocks), dtype=torch.uint8)
    if scales is None:
        scales = x.new_empty((rows, blocks), dtype=torch.uint8)
    pc, ps = _bytes(codes, "codes", (rows, 16 * blocks)), _bytes(scales, "scales", (rows, blocks))
    binding._check(lib.ts_mx_quantize(px, _DTYPES[x.dtype], rows, cols, stride, pc, ps, _stream(x)))
    return codes, scales


def ts_mx_dequantize(codes, scales, cols, dtype=torch.float32, out=None):
    """The values [rows][cols] that codes and scales stand for (exact in both types; infinite from 2^128 on)."""
    lib = _lib or _load()
    if dtype not in _DTYPES:
        raise TypeError("dtype: float32 or bfloat16 is needed, got %s" % dtype)
    rows, blocks = codes.shape[0], (cols + 31) // 32
    pc, ps = _bytes(codes, "codes", (rows, 16 * blocks)), _bytes(scales, "scales", (rows, blocks))
    if out is None:
        out = codes.new_empty((rows, cols), dtype=dtype)
    po, stride = _rows(out, "out", cols, dtype)
    if out.shape[0] != rows:
        _refuse("out: %d rows are needed, got %d", rows, out.shape[0])
    binding._check(lib.ts_mx_dequantize(pc, ps, rows, cols, po, _DTYPES[dtype], stride, _stream(codes)))
    return out


def ts_mx_packed_bytes(n_out, n_in):
    n = C.c_uint64()
    binding._check(_load().ts_mx_packed_bytes(_int(n_out, "n_out"), _int(n_in, "n_in"), C.byref(n)))
    return n.value


def ts_mx_pack(codes, scales, n_in, out=None):
    """Weights [n_out][n_in], given as codes and scales, laid out for ts_mx_project: a uint8 tensor to keep.  The tensor object carries
    the sizes (`ts_mx_shape`), which ts_mx_project holds its call against; of a copy or a view without them only the bytes are checked."""
    lib = _lib or _load()
    n_out, blocks = codes.shape[0], (n_in + 31) // 32
    pc, ps = _bytes(codes, "codes", (n_out, 16 * blocks)), _bytes(scales, "scales", (n_out, blocks))
    n = ts_mx_packed_bytes(n_out, n_in)
    if out is None:
        out = torch.empty(n, dtype=torch.uint8, device=codes.device)
    binding._check(lib.ts_mx_pack(pc, ps, n_out, n_in, _bytes(out, "out", (n,)), _stream(codes)))
    out.ts_mx_shape = (n_out, n_in)
    return out


def ts_mx_project(packed, n_out, x, out=None):
    """x [rows][n_in] times the packed weights' transpose: [rows][n_out] in x's type."""
    lib = _lib or _load()
    px, xs = _rows(x, "x")
    rows, n_in = x.shape
    pw = _bytes(packed, "packed")
    if n_in < 1 or n_out < 1 or packed.numel() != -(-n_out // 16) * -(-n_in // 128) * _RECORD or getattr(packed, "ts_mx_shape", (n_out, n_in)) != (n_out, n_in):
        _refuse("packed: not the weights of a [%d][%d] matrix", n_out, n_in)
    if out is None:
        out = x.new_empty((rows, n_out))
        po, os_ = out.data_ptr(), n_out
    else:
        po, os_ = _rows(out, "out", n_out, x.dtype)
        if out.shape[0] != rows:
            _refuse("out: %d rows are needed, got %d", rows, out.shape[0])
    binding._check(lib.ts_mx_project(pw, n_out, n_in, px, _DTYPES[x.dtype], rows, xs, po, os_, _stream(x)))
    return out


# ---- one layer of a paged cache -----------------------------------------------------------
def ts_kv_layer_pages(kv, layer):
    """The pages of one layer of a library cache, to be given to ts_kv_append / ts_kv_attend as `k_pages` (with v_pages None)."""
    p = ts_kv_pages()
    binding._check(_load().ts_kv_layer_pages(kv, _int(layer, "layer"), C.byref(p)))
    return p


def ts_kv_page_table(kv, capacity_tokens):
    """The cache's physical pages in order: numpy int32 [ceil(capacity_tokens / 16)], of the capacity it was allocated with."""
    out = np.empty((capacity_tokens + TS_PAGE_SIZE - 1) // TS_PAGE_SIZE, np.int32)
    binding._check(_load().ts_kv_page_table(kv, out.ctypes.data_as(C.POINTER(C.c_int32)), len(out)))
    return out


def ts_kv_extend(kv, n_pos, stream=None):
    """Counts n_pos positions that were appended on `stream` (a torch stream of the cache's GPU; default: the current one) as committed."""
    s = (stream or torch.cuda.current_stream()).cuda_stream
    binding._check(_load().ts_kv_extend(kv, _int(n_pos, "n_pos"), s))


def _pages(k_pages, v_pages):
    """The members of a ts_kv_pages."""
    if v_pages is None:
        if not isinstance(k_pages, ts_kv_pages):
            raise TypeError("v_pages is missing")
        return k_pages.k or 0, k_pages.v or 0, k_pages.n_pages, k_pages.n_kv_heads, k_pages.head_dim, k_pages.dtype
    ks = k_pages.shape
    if len(ks) != 4 or ks[2] != TS_PAGE_SIZE or not k_pages.is_contiguous() or not v_pages.is_contiguous() or not k_pages.is_cuda or not v_pages.is_cuda:
        _refuse("k_pages: a contiguous [pages][heads][%d][head_dim] tensor on a GPU is needed, got %s", TS_PAGE_SIZE, tuple(ks))
    n, h, _, hd = ks
    if v_pages.shape != (n, h, hd, TS_PAGE_SIZE):
        _refuse("v_pages: shape %s is needed, got %s", (n, h, hd, TS_PAGE_SIZE), tuple(v_pages.shape))
    dtype = k_pages.dtype
    if dtype not in _DTYPES or v_pages.dtype != dtype:
        raise TypeError("pages: float32 or bfloat16 are needed, got %s and %s" % (dtype, v_pages.dtype))
    if k_pages.requires_grad or v_pages.requires_grad:
        _no_gradient("pages")
    return k_pages.data_ptr(), v_pages.data_ptr(), n, h, hd, _DTYPES[dtype]


def _table(t, n_seqs):
    shape, strides = t.shape, t.stride()
    if len(shape) != 2 or t.dtype is not torch.int32 or not t.is_cuda or shape[0] < n_seqs or shape[1] < 1 or (strides[1] != 1 and shape[1] > 1) or (strides[0] < shape[1] and shape[0] > 1):
        _refuse("table: int32 [%d][pages] on a GPU is needed, got %s %s", n_seqs, t.dtype, tuple(shape))
    return t.data_ptr(), strides[0] if strides[0] > shape[1] else shape[1], shape[1]


def ts_kv_append(k_pages, v_pages, table, lengths, row_offsets, q, k, v, rope_theta, q_out=None):
    """Rows of k and v ([rows][kv heads * head_dim]) into the cache at lengths[s], lengths[s] + 1, ... of their sequences, keys
    rotated; with q ([rows][heads * head_dim]) the rotated queries, which are returned.  See the header."""
    lib = _lib or _load()
    pages = _pages(k_pages, v_pages)
    n, kv_heads, hd = row_offsets.shape[0] - 1, pages[3], pages[4]
    table, t_stride, t_width = _table(table, n)
    width = kv_heads * hd
    pk, k_stride = _rows(k, "k", width)
    dtype, rows = k.dtype, k.shape[0]
    pv, v_stride = _rows(v, "v", width, dtype)
    if v.shape[0] != rows:
        _refuse("v: %d rows are needed, got %d", rows, v.shape[0])
    pq, q_stride, po, o_stride, heads = 0, 0, 0, 0, 0
    if q is not None:
        pq, q_stride = _rows(q, "q", None, dtype)
        q_rows, q_width = q.shape
        if q_rows != rows or q_width < 1 or q_width % hd:
            _refuse("q: %d rows of a multiple of %d values are needed, got %s", rows, hd, tuple(q.shape))
        if q_out is None:
            q_out = torch.zeros(q.shape, dtype=dtype, device=q.device)
        po, o_stride = _rows(q_out, "q_out", q_width, dtype)
        if q_out.shape[0] != rows:
            _refuse("q_out: %d rows are needed, got %d", rows, q_out.shape[0])
        heads = q_width // hd
    elif q_out is not None:
        _refuse("q_out without q")
    try:
        a = _pack_append(*pages, table, t_stride, t_width, _ints(lengths, "lengths", n), _ints(row_offsets, "row_offsets", 2), n, rows, heads, _DTYPES[dtype],
                         pq, q_stride, pk, k_stride, pv, v_stride, po, o_stride, rope_theta)
    except struct.error as e:                              # a number that its member cannot hold
        _out_of_range(e)
    binding._check(lib.ts_kv_append(a, _stream(k)))
    return q_out


def ts_kv_attend_workspace(n_seqs, n_q_heads, n_kv_heads, head_dim, max_len, window=0, device="cuda"):
    """A workspace tensor for ts_kv_attend calls of these sizes (None where they need none)."""
    n = C.c_uint64()
    sizes = [_int(v, name) for v, name in ((n_seqs, "n_seqs"), (n_q_heads, "n_q_heads"), (n_kv_heads, "n_kv_heads"), (head_dim, "head_dim"),
                                           (max_len, "max_len"), (window, "window"))]
    binding._check(_load().ts_kv_attend_workspace(*sizes, C.byref(n)))
    return torch.empty(n.value, dtype=torch.uint8, device=device) if n.value else None


def _given_lse(t, n, heads):
    if t.shape != (n, heads) or t.dtype is not torch.float32 or not t.is_contiguous() or not t.is_cuda:
        _refuse("lse: a contiguous fp32 [%d][%d] tensor on a GPU is needed, got %s %s", n, heads, t.dtype, tuple(t.shape))
    if t.requires_grad:
        _no_gradient("lse")


def ts_kv_attend(k_pages, v_pages, table, lengths, q, max_len, window=0, scale=None, workspace=None, out=None, lse=None):
    """Attention of one token per sequence, q [n_seqs][heads * head_dim]: (out like q, lse fp32 [n_seqs][heads]).  scale None:
    1 / sqrt(head_dim).  workspace: of ts_kv_attend_workspace; without one the call allocates it.  See the header."""
    lib = _lib or _load()
    pages = _pages(k_pages, v_pages)
    kv_heads, hd = pages[3], pages[4]
    pq, q_stride = _rows(q, "q")
    n, width = q.shape
    if n < 1 or width < 1 or width % hd:
        _refuse("q: rows of a multiple of %d values are needed, got %s", hd, tuple(q.shape))
    table, t_stride, t_width = _table(table, n)
    heads, dtype = width // hd, q.dtype
    if out is None:
        out = q.new_empty((n, width))
        po, o_stride = out.data_ptr(), width
    else:
        po, o_stride = _rows(out, "out", width, dtype)
    if lse is None:
        lse = q.new_empty((n, heads), dtype=torch.float32)
    else:
        _given_lse(lse, n, heads)
    if out.shape[0] != n:
        _refuse("out: %d rows are needed, got %d", n, out.shape[0])
    if workspace is None:
        workspace = ts_kv_attend_workspace(n, heads, kv_heads, hd, max_len, window, q.device)
    ws, ws_bytes = (0, 0) if workspace is None else (_bytes(workspace, "workspace"), workspace.numel())
    try:
        a = _pack_attend(*pages, table, t_stride, t_width, _ints(lengths, "lengths", n), n, max_len, window, heads, _DTYPES[dtype], pq, q_stride, po, o_stride,
                         lse.data_ptr(), hd ** -0.5 if scale is None else scale, ws, ws_bytes)
    except struct.error as e:
        _out_of_range(e)
    binding._check(lib.ts_kv_attend(a, _stream(q)))
    return out, lse


# ---- more rows, other rotations, 8-bit pages ----------------------------------------------
def _any_pages(k_pages, v_pages, scales):
    """The members of a ts_kv_pages_any: pages of fp32 or bf16 (or a library cache's layer) without scales, or of float8_e4m3fn with (k_scales, v_scales)."""
    if v_pages is None or k_pages.dtype is not torch.float8_e4m3fn:
        if scales is not None:
            _refuse("scales belong to float8_e4m3fn pages")
        return _pages(k_pages, v_pages) + (0, 0)
    ks = k_pages.shape
    if len(ks) != 4 or ks[2] != TS_PAGE_SIZE or not k_pages.is_contiguous() or not v_pages.is_contiguous() or not k_pages.is_cuda or not v_pages.is_cuda:
        _refuse("k_pages: a contiguous [pages][heads][%d][head_dim] tensor on a GPU is needed, got %s", TS_PAGE_SIZE, tuple(ks))
    n, h, _, hd = ks
    if v_pages.shape != (n, h, hd, TS_PAGE_SIZE):
        _refuse("v_pages: shape %s is needed, got %s", (n, h, hd, TS_PAGE_SIZE), tuple(v_pages.shape))
    if v_pages.dtype is not torch.float8_e4m3fn:
        raise TypeError("pages: two of one type are needed, got %s and %s" % (k_pages.dtype, v_pages.dtype))
    if k_pages.requires_grad or v_pages.requires_grad:
        _no_gradient("pages")
    if scales is None or len(scales) != 2:
        _refuse("scales: (k_scales, v_scales) are needed with float8_e4m3fn pages")
    shape = (n, h, TS_PAGE_SIZE)
    return k_pages.data_ptr(), v_pages.data_ptr(), n, h, hd, TS_DTYPE_E4M3, _bytes(scales[0], "k_scales", shape), _bytes(scales[1], "v_scales", shape)


def _gain(t, name, hd, dtype):
    if t is None:
        return 0
    if t.dtype not in _DTYPES or (dtype is not None and t.dtype is not dtype):
        raise TypeError("%s: %s is needed, got %s" % (name, dtype or "float32 or bfloat16", t.dtype))
    if t.shape != (hd,) or not t.is_contiguous() or not t.is_cuda:
        _refuse("%s: %d contiguous values on a GPU are needed, got %s", name, hd, tuple(t.shape))
    if t.requires_grad:
        _no_gradient(name)
    return t.data_ptr()


def ts_kv_append_norm_rope(k_pages, v_pages, table, lengths, row_offsets, q, k, v, rope_theta=0.0, rope_dim=None, rope_pairs=False, rope_freqs=None,
                           rope_magnitude=1.0, q_norm=None, k_norm=None, norm_eps=1e-6, positions=None, scales=None, q_out=None):
    """ts_kv_append with norms of the heads (gains q_norm, k_norm [head_dim]), rotations of the first rope_dim values (None: all) in halves or
    neighbouring pairs, by theta or a table rope_freqs (fp32 [rope_dim / 2], radians per position), at the rows' positions or at given ones
    (int32 [rows]), and into pages of any type (float8_e4m3fn pages: scales = (k_scales, v_scales), uint8 [pages][heads][16]).  Returns
    the queries as rotated (q_out; zeros where a row belongs to no sequence).  See the header."""
    lib = _lib or _load()
    pages = _any_pages(k_pages, v_pages, scales)
    n, kv_heads, hd = row_offsets.shape[0] - 1, pages[3], pages[4]
    table, t_stride, t_width = _table(table, n)
    width = kv_heads * hd
    pk, k_stride = _rows(k, "k", width)
    dtype, rows = k.dtype, k.shape[0]
    pv, v_stride = _rows(v, "v", width, dtype)
    if v.shape[0] != rows:
        _refuse("v: %d rows are needed, got %d", rows, v.shape[0])
    pq, q_stride, po, o_stride, heads = 0, 0, 0, 0, 0
    if q is not None:
        pq, q_stride = _rows(q, "q", None, dtype)
        q_rows, q_width = q.shape
        if q_rows != rows or q_width < 1 or q_width % hd:
            _refuse("q: %d rows of a multiple of %d values are needed, got %s", rows, hd, tuple(q.shape))
        if q_out is None:
            q_out = torch.zeros(q.shape, dtype=dtype, device=q.device)
        po, o_stride = _rows(q_out, "q_out", q_width, dtype)
        if q_out.shape[0] != rows:
            _refuse("q_out: %d rows are needed, got %d", rows, q_out.shape[0])
        heads = q_width // hd
    elif q_out is not None or q_norm is not None:
        _refuse("q_out or q_norm without q")
    if rope_dim is None:
        rope_dim = hd
    norm_type = q_norm.dtype if q_norm is not None else None
    pqn, pkn = _gain(q_norm, "q_norm", hd, None), _gain(k_norm, "k_norm", hd, norm_type)
    if k_norm is not None:
        norm_type = k_norm.dtype
    freqs = 0
    if rope_freqs is not None:
        if rope_freqs.dtype is not torch.float32 or not rope_freqs.is_cuda or rope_freqs.dim() != 1 or not rope_freqs.is_contiguous() or rope_freqs.shape[0] * 2 != rope_dim:
            _refuse("rope_freqs: %d contiguous fp32 on a GPU are needed, got %s %s", rope_dim // 2, rope_freqs.dtype, tuple(rope_freqs.shape))
        if rope_freqs.requires_grad:
            _no_gradient("rope_freqs")
        freqs = rope_freqs.data_ptr()
    try:
        a = _pack_append_norm_rope(*pages, table, t_stride, t_width, _ints(lengths, "lengths", n), _ints(row_offsets, "row_offsets", 2),
                                   0 if positions is None else _ints(positions, "positions", rows), n, rows, heads, _DTYPES[dtype], pq, q_stride, pk, k_stride,
                                   pv, v_stride, po, o_stride, pqn, pkn, _DTYPES.get(norm_type, 0), norm_eps, freqs, rope_theta, rope_magnitude, rope_dim, bool(rope_pairs))
    except (struct.error, OverflowError) as e:             # a number that its member cannot hold
        _out_of_range(e)
    binding._check(lib.ts_kv_append_norm_rope(a, _stream(k)))
    return q_out


def _read_into(t, name, n_rows, width, dtype):
    if t is None:
        return 0, 0
    at = _rows(t, name, width, dtype)
    if t.shape[0] != n_rows:
        _refuse("%s: %d rows are needed, got %d", name, n_rows, t.shape[0])
    return at


def ts_kv_read(k_pages, v_pages, table, starts, row_offsets, n_rows, dtype=torch.bfloat16, scales=None, k_out=None, v_out=None):
    """Positions starts[s], starts[s] + 1, ... of each sequence as rows row_offsets[s], ...: (k, v), [n_rows][heads * head_dim] of `dtype`, zeros where a
    row is no position.  starts None: from 0 on.  With k_out and / or v_out (of `dtype`) only those are written.  See the header."""
    lib = _lib or _load()
    if dtype not in _DTYPES:
        raise TypeError("dtype: float32 or bfloat16 is needed, got %s" % dtype)
    pages = _any_pages(k_pages, v_pages, scales)
    n, width = row_offsets.shape[0] - 1, pages[3] * pages[4]
    p_table, t_stride, t_width = _table(table, n)
    if n_rows < 0:
        _refuse("n_rows: %d", n_rows)
    own = k_out is None and v_out is None
    if own:
        k_out, v_out = table.new_empty((n_rows, width), dtype=dtype), table.new_empty((n_rows, width), dtype=dtype)
        at = (k_out.data_ptr(), width, v_out.data_ptr(), width)
    else:
        at = _read_into(k_out, "k_out", n_rows, width, dtype) + _read_into(v_out, "v_out", n_rows, width, dtype)
    try:
        a = _pack_read(*pages, p_table, t_stride, t_width, 0 if starts is None else _ints(starts, "starts", n), _ints(row_offsets, "row_offsets", 2), n, n_rows,
                       _DTYPES[dtype], own, *at)
    except struct.error as e:
        _out_of_range(e)
    binding._check(lib.ts_kv_read(a, _stream(table)))
    return k_out, v_out


def ts_kv_attend_rows_workspace(n_seqs, n_rows, n_q_heads, n_kv_heads, head_dim, max_len, window=0, device="cuda"):
    """A workspace tensor for ts_kv_attend_rows calls of these sizes (None where they need none)."""
    n = C.c_uint64()
    sizes = [_int(v, name) for v, name in ((n_seqs, "n_seqs"), (n_rows, "n_rows"), (n_q_heads, "n_q_heads"), (n_kv_heads, "n_kv_heads"), (head_dim, "head_dim"),
                                           (max_len, "max_len"), (window, "window"))]
    binding._check(_load().ts_kv_attend_rows_workspace(*sizes, C.byref(n)))
    return torch.empty(n.value, dtype=torch.uint8, device=device) if n.value else None


def ts_kv_attend_rows(k_pages, v_pages, table, lengths, row_offsets, q, max_len, window=0, scale=None, ancestors=None, scales=None, workspace=None,
                      out=None, lse=None):
    """Attention of the rows of chunks, q [rows][heads * head_dim], over a cache of any type that holds them at lengths[s], lengths[s] + 1, ...:
    (out like q, lse fp32 [rows][heads]; allocated ones are zeros where a row belongs to no sequence).  row_offsets None: one row a sequence.
    ancestors: int64 [rows], the sets of a draft tree.  scale None: 1 / sqrt(head_dim).  workspace: of ts_kv_attend_rows_workspace; without one the
    call allocates it.  See the header."""
    lib = _lib or _load()
    pages = _any_pages(k_pages, v_pages, scales)
    kv_heads, hd = pages[3], pages[4]
    pq, q_stride = _rows(q, "q")
    rows, width = q.shape
    if width < 1 or width % hd:
        _refuse("q: rows of a multiple of %d values are needed, got %s", hd, tuple(q.shape))
    n = rows if row_offsets is None else row_offsets.shape[0] - 1
    table, t_stride, t_width = _table(table, n)
    heads, dtype = width // hd, q.dtype
    if out is None:
        out = q.new_empty((rows, width)) if row_offsets is None else q.new_zeros((rows, width))
    po, o_stride = _rows(out, "out", width, dtype)
    if out.shape[0] != rows:
        _refuse("out: %d rows are needed, got %d", rows, out.shape[0])
    if lse is None:
        lse = q.new_empty((rows, heads), dtype=torch.float32) if row_offsets is None else q.new_zeros((rows, heads), dtype=torch.float32)
    else:
        _given_lse(lse, rows, heads)
    sets = 0
    if ancestors is not None:
        if ancestors.dtype is not torch.int64 or not ancestors.is_cuda or ancestors.dim() != 1 or not ancestors.is_contiguous() or ancestors.shape[0] < rows:
            _refuse("ancestors: at least %d contiguous int64 on a GPU are needed, got %s %s", rows, ancestors.dtype, tuple(ancestors.shape))
        sets = ancestors.data_ptr()
    if workspace is None:
        workspace = ts_kv_attend_rows_workspace(n, rows, heads, kv_heads, hd, max_len, window, q.device)
    ws, ws_bytes = (0, 0) if workspace is None else (_bytes(workspace, "workspace"), workspace.numel())
    try:
        a = _pack_rows(*pages, table, t_stride, t_width, _ints(lengths, "lengths", n), 0 if row_offsets is None else _ints(row_offsets, "row_offsets", 2), sets,
                       n, rows, max_len, window, heads, _DTYPES[dtype], pq, q_stride, po, o_stride, lse.data_ptr(), hd ** -0.5 if scale is None else scale, ws, ws_bytes)
    except (struct.error, OverflowError) as e:
        _out_of_range(e)
    binding._check(lib.ts_kv_attend_rows(a, _stream(q)))
    return out, lse
