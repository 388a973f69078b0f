"""Python binding of the attention operators of libopattr (include/opattr_attn.h).

Argument marshalling only, as in ``opattr``: torch device tensors are handed to
the C entry points by pointer, outputs are written where the caller says (or
into new tensors), and the work goes to the current HIP stream. There is no CPU
fallback: a missing library raises.

Tensors of queries, keys, values, outputs and gradients are [tokens, heads,
head_dim] in bfloat16 or float16, any strides with the last one 1 (multiples of
8 elements, 16-byte aligned). Lengths, offsets and page tables are contiguous
int32 tensors. Data errors go to the ``diag`` record, if one is given
(``new_diag``; read it with ``opattr.read_diag``).
"""
from __future__ import annotations

import ctypes as C
import math
import struct
import threading

import torch

from . import opattr
from .opattr import Outputs, Workspace  # noqa: F401  (part of this interface)

BF16, F16 = 0, 1
MAX_HEAD_DIM, MAX_PAGED_GROUP, MAX_PAGE_SIZE = 128, 16, 1024


class opattr_rows(C.Structure):
    _fields_ = [("p", C.c_void_p), ("token_stride", C.c_int64), ("head_stride", C.c_int64)]


class opattr_attn_shape(C.Structure):
    _fields_ = [("n_q", C.c_int64), ("n_k", C.c_int64), ("cu_q", C.c_void_p),
                ("cu_k", C.c_void_p), ("n_seqs", C.c_int32), ("n_heads", C.c_int32),
                ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("dtype", C.c_int32),
                ("causal", C.c_int32), ("scale", C.c_float)]


class opattr_kv_pages(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("page_stride", C.c_int64),
                ("token_stride", C.c_int64), ("head_stride", C.c_int64), ("n_pages", C.c_int32),
                ("page_size", C.c_int32), ("table", C.c_void_p), ("n_seqs", C.c_int32),
                ("table_stride", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("dtype", C.c_int32)]


class opattr_page_pool(C.Structure):
    _fields_ = [("data", C.c_void_p), ("plane_stride", C.c_int64), ("page_stride", C.c_int64),
                ("n_planes", C.c_int32), ("n_pages", C.c_int32), ("page_bytes", C.c_int32),
                ("page_size", C.c_int32), ("held", C.c_void_p)]


EXPORTS = ("opattr_attn_prompt", "opattr_attn_prompt_grad",
           "opattr_attn_prompt_grad_workspace_bytes", "opattr_attn_paged",
           "opattr_attn_paged_workspace_bytes", "opattr_kv_append", "opattr_pages_fork",
           "opattr_pages_fork_workspace_bytes", "opattr_pages_compact",
           "opattr_pages_compact_workspace_bytes")

_lib = None
_call = {}


class _Args(threading.local):
    """The structs of one call, side by side in a buffer of the calling thread's:
    written by one struct.pack and passed by address, which costs a fraction of
    building a ctypes Structure for each."""

    def __init__(self, *structs):
        self.pack_into = struct.Struct("".join(_FORMAT[c] for c in structs)).pack_into
        self.buf = C.create_string_buffer(sum(C.sizeof(c) for c in structs))
        at, self.at = C.addressof(self.buf), []
        for c in structs:
            self.at.append(at)
            at += C.sizeof(c)

    def set(self, *values):
        self.pack_into(self.buf, 0, *values)
        return self.at


_FORMAT = {opattr_rows: "Pqq", opattr_attn_shape: "qqPPiiiiiif4x",
           opattr_kv_pages: "PPqqqiiPiiiii4x", opattr_page_pool: "PqqiiiiP"}
_PROMPT = _Args(opattr_attn_shape, *[opattr_rows] * 4)
_GRAD = _Args(opattr_attn_shape, *[opattr_rows] * 8)
_PAGED = _Args(opattr_kv_pages, opattr_rows, opattr_rows)
_POOL = _Args(opattr_page_pool)


def library():
    """libopattr with the attention entry points declared."""
    global _lib
    if _lib is not None:
        return _lib
    L = opattr.library()
    P, vp, i32, i64, sz = C.POINTER, C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
    rows = P(opattr_rows)
    L.opattr_attn_prompt.argtypes = [P(opattr_attn_shape), rows, rows, rows, rows, vp, vp, vp]
    L.opattr_attn_prompt_grad_workspace_bytes.argtypes = [P(opattr_attn_shape)]
    L.opattr_attn_prompt_grad.argtypes = [P(opattr_attn_shape), rows, rows, rows, rows, rows, vp,
                                          rows, rows, rows, vp, vp, sz, vp]
    L.opattr_attn_paged_workspace_bytes.argtypes = [P(opattr_kv_pages), i32]
    L.opattr_attn_paged.argtypes = [P(opattr_kv_pages), i32, rows, vp, C.c_float, rows, vp, vp,
                                    vp, sz, vp]
    L.opattr_kv_append.argtypes = [P(opattr_kv_pages), i64, vp, rows, rows, vp, vp, vp, vp]
    L.opattr_pages_fork_workspace_bytes.argtypes = [i32, i32, i32, i32]
    L.opattr_pages_fork.argtypes = [P(opattr_page_pool), vp, vp, i32, i32, vp, vp, i32, vp, vp,
                                    vp, vp, vp, sz, vp]
    L.opattr_pages_compact_workspace_bytes.argtypes = [i32]
    L.opattr_pages_compact.argtypes = [P(opattr_page_pool), vp, i32, i32, vp, vp, vp, vp, vp, sz,
                                       vp]
    for f in EXPORTS:
        getattr(L, f).restype = sz if f.endswith("_bytes") else C.c_int
        # the same entry point taking its structs by address
        _call[f] = L[f]
        _call[f].restype = getattr(L, f).restype
        _call[f].argtypes = [vp if isinstance(t, type(rows)) else t for t in getattr(L, f).argtypes]
    _lib = L
    return L


def _entry(name):
    if _lib is None:
        library()
    return _call[name]


def new_diag(device="cuda:0", stream=None):
    """A cleared diag record on the device."""
    return opattr._new_diag(device, stream)


def _dtype(t):
    d = t.dtype
    if t.get_device() < 0:
        raise TypeError("device tensors are taken")
    if d is torch.bfloat16:
        return BF16
    if d is torch.float16:
        return F16
    raise TypeError(f"bfloat16 or float16 tensors are taken, not {d}")


def _rows(t, like, shape, name):
    """The opattr_rows of a [tokens, heads, head_dim] tensor of like's type."""
    if t.dtype is not like.dtype or t.get_device() != like.get_device():
        raise TypeError(f"{name}: {t.dtype} on {t.device}, expected {like.dtype} on {like.device}")
    if t.shape != shape:
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {tuple(shape)}")
    ts, hs, es = t.stride()
    n, heads, d = shape
    if es != 1 and d > 1:
        raise ValueError(f"{name}: the last dimension's values must lie side by side")
    # the stride of a single row or head says nothing
    return t.data_ptr(), ts if n > 1 else d, hs if heads > 1 else 0


def _array(t, dtype, like, shape, name):
    """The address of a contiguous array."""
    if t.dtype is not dtype or t.get_device() != like.get_device() or not t.is_contiguous():
        raise TypeError(f"{name}: a contiguous {dtype} tensor on {like.device} is wanted")
    if t.shape != shape:
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {shape}")
    return t.data_ptr()


def _shape(q, k, cu_q, cu_k, causal, scale):
    if q.dim() != 3 or k.dim() != 3 or cu_q.dim() != 1:
        raise ValueError("queries and keys are [tokens, heads, head_dim], offsets one more than "
                         "sequences")
    n_q, heads, d = q.shape
    n_k, kv_heads, _ = k.shape
    n = cu_q.shape[0]
    p = _array(cu_q, torch.int32, q, (n,), "cu_q")
    return (n_q, n_k, p, p if cu_k is cu_q else _array(cu_k, torch.int32, q, (n,), "cu_k"), n - 1,
            heads, kv_heads, d, _dtype(q), 1 if causal else 0,
            1.0 / math.sqrt(d) if scale is None else scale)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream(stream, on, *made):
    """The stream's handle: the caller's, or the current one of `on`'s device.
    Tensors that a call made itself belong to the current stream: one used on
    another is kept until that has passed the call."""
    if stream is None:
        # current_stream() builds a Stream object for it: 4 us a call
        return torch._C._cuda_getCurrentRawStream(on.get_device())
    for t in made:
        t.record_stream(stream)
    return stream.cuda_stream


def opattr_attn_prompt(q, k, v, cu_q, cu_k=None, causal=True, scale=None, out=None, lse=None,
                       diag=None, stream=None):
    """Attention over packed prompts: (out, lse). Sequence b has queries
    q[cu_q[b]:cu_q[b+1]] and keys k[cu_k[b]:cu_k[b+1]] (cu_k None: as cu_q);
    scale None: 1 / sqrt(head_dim). Rows of ``out`` and ``lse`` outside every
    sequence are not written."""
    call = _entry("opattr_attn_prompt")
    a = _shape(q, k, cu_q, cu_q if cu_k is None else cu_k, causal, scale)
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    rows = (a[5], a[0])
    if lse is None:
        lse = torch.empty(rows, dtype=torch.float32, device=q.device)
    qs, ks = q.shape, (a[1], a[6], a[7])
    at = _PROMPT.set(*a, *_rows(q, q, qs, "q"), *_rows(k, q, ks, "k"), *_rows(v, q, ks, "v"),
                     *_rows(out, q, qs, "out"))
    rc = call(*at, _array(lse, torch.float32, q, rows, "lse"), _ptr(diag),
              _stream(stream, q, out, lse))
    if rc:
        opattr._check(rc, "opattr_attn_prompt")
    return out, lse


def opattr_attn_prompt_grad(dout, q, k, v, out, lse, cu_q, cu_k=None, causal=True, scale=None,
                            dq=None, dk=None, dv=None, ws: Workspace | None = None, diag=None,
                            stream=None):
    """Gradients of sum(out * dout): (dq, dk, dv). out and lse are
    opattr_attn_prompt's for the same inputs."""
    call, size = _entry("opattr_attn_prompt_grad"), _call["opattr_attn_prompt_grad_workspace_bytes"]
    a = _shape(q, k, cu_q, cu_q if cu_k is None else cu_k, causal, scale)
    if dq is None:
        dq = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    if dk is None:
        dk = torch.empty(k.shape, dtype=q.dtype, device=q.device)
    if dv is None:
        dv = torch.empty(k.shape, dtype=q.dtype, device=q.device)
    qs, ks = q.shape, (a[1], a[6], a[7])
    at = _GRAD.set(*a, *_rows(dout, q, qs, "dout"), *_rows(q, q, qs, "q"), *_rows(k, q, ks, "k"),
                   *_rows(v, q, ks, "v"), *_rows(out, q, qs, "out"), *_rows(dq, q, qs, "dq"),
                   *_rows(dk, q, ks, "dk"), *_rows(dv, q, ks, "dv"))
    buf = (ws or Workspace(q.device)).get(size(at[0]))
    rc = call(*at[:6], _array(lse, torch.float32, q, (a[5], a[0]), "lse"), *at[6:], _ptr(diag),
              buf.data_ptr(), buf.numel(), _stream(stream, q, buf, dq, dk, dv))
    if rc:
        opattr._check(rc, "opattr_attn_prompt_grad")
    return dq, dk, dv


def _kv_pages(k_pages, v_pages, table):
    """The values of an opattr_kv_pages."""
    strides = k_pages.stride()
    if k_pages.dim() != 4 or k_pages.shape != v_pages.shape or strides != v_pages.stride() or \
            k_pages.dtype is not v_pages.dtype or k_pages.get_device() != v_pages.get_device():
        raise ValueError("k_pages and v_pages are [pages, page_size, kv_heads, head_dim], alike "
                         "in shape, strides and type")
    n, size, heads, d = k_pages.shape
    ps, ts, hs, es = strides
    if es != 1 and d > 1:
        raise ValueError("k_pages: the last dimension's values must lie side by side")
    if table.dim() != 2:
        raise ValueError("table is [sequences, entries]")
    b, width = table.shape
    return (k_pages.data_ptr(), v_pages.data_ptr(), ps if n > 1 else 0, ts if size > 1 else 0,
            hs if heads > 1 else 0, n, size,
            _array(table, torch.int32, k_pages, (b, width), "table"), b, width, heads, d,
            _dtype(k_pages))


def opattr_attn_paged(q, k_pages, v_pages, table, lens, scale=None, out=None, lse=None,
                      ws: Workspace | None = None, diag=None, stream=None):
    """Attention of one token a sequence, q [sequences, heads, head_dim], over
    the first lens[b] tokens of each: (out, lse [heads, sequences])."""
    call, size = _entry("opattr_attn_paged"), _call["opattr_attn_paged_workspace_bytes"]
    c = _kv_pages(k_pages, v_pages, table)
    b, d = c[8], c[11]
    if q.dtype is not k_pages.dtype or q.dim() != 3 or q.shape[2] != d:
        raise ValueError("q: not [sequences, heads, head_dim] of the cache's type")
    h = q.shape[1]
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    if lse is None:
        lse = torch.empty((h, b), dtype=torch.float32, device=q.device)
    shape = (b, h, d)
    at = _PAGED.set(*c, *_rows(q, k_pages, shape, "q"), *_rows(out, q, shape, "out"))
    buf = (ws or Workspace(q.device)).get(size(at[0], h))
    rc = call(at[0], h, at[1], _array(lens, torch.int32, q, (b,), "lens"),
              1.0 / math.sqrt(d) if scale is None else scale, at[2],
              _array(lse, torch.float32, q, (h, b), "lse"), _ptr(diag), buf.data_ptr(),
              buf.numel(), _stream(stream, q, buf, out, lse))
    if rc:
        opattr._check(rc, "opattr_attn_paged")
    return out, lse


def opattr_kv_append(k_new, v_new, cu, k_pages, v_pages, table, lens, lens_out=None, diag=None,
                     stream=None):
    """Rows cu[b] .. cu[b+1] of k_new and v_new become the next tokens of
    sequence b, which holds lens[b]; returns the new lengths."""
    call = _entry("opattr_kv_append")
    c = _kv_pages(k_pages, v_pages, table)
    n, b = k_new.shape[0], c[8]
    if lens_out is None:
        lens_out = torch.empty(b, dtype=torch.int32, device=k_pages.device)
    shape = (n, c[10], c[11])
    at = _PAGED.set(*c, *_rows(k_new, k_pages, shape, "k_new"),
                    *_rows(v_new, k_pages, shape, "v_new"))
    rc = call(at[0], n, _array(cu, torch.int32, k_pages, (b + 1,), "cu"), at[1], at[2],
              _array(lens, torch.int32, k_pages, (b,), "lens"),
              _array(lens_out, torch.int32, k_pages, (b,), "lens_out"), _ptr(diag),
              _stream(stream, k_pages, lens_out))
    if rc:
        opattr._check(rc, "opattr_kv_append")
    return lens_out


def _pool(pool, page_size, held):
    """The values of the opattr_page_pool of a [planes, pages, ...] tensor whose
    pages lie in one piece each."""
    if pool.dim() < 3:
        raise ValueError("pool is [planes, pages, ...]")
    if pool.get_device() < 0:
        raise TypeError("device tensors are taken")
    shape, strides = pool.shape, pool.stride()
    each = 1
    for n, s in zip(shape[:1:-1], strides[:1:-1]):
        if n > 1 and s != each:
            raise ValueError("a page's values must lie side by side")
        each *= n
    size = pool.element_size()
    planes, pages = shape[:2]
    return (pool.data_ptr(), strides[0] * size if planes > 1 else 0,
            strides[1] * size if pages > 1 else each * size, planes, pages, each * size,
            page_size, 0 if held is None else _array(held, torch.int32, pool, (pages,), "held"))


def opattr_pages_fork(pool, page_size, table, lens, parent, room=None, held=None, table_out=None,
                      lens_out=None, refs=None, ws: Workspace | None = None, diag=None,
                      stream=None) -> Outputs:
    """The next page table: row i continues row parent[i] (-1: empty), with room
    for room[i] tokens. pool [planes, pages, ...] holds the pages that a forked
    row's last, part-filled page is copied in. Returns table, lens and refs."""
    call, size = _entry("opattr_pages_fork"), _call["opattr_pages_fork_workspace_bytes"]
    if table.dim() != 2 or parent.dim() != 1:
        raise ValueError("table is [rows, entries], parent [rows of the next table]")
    p = _pool(pool, page_size, held)
    (rows, width), n, pages = table.shape, parent.shape[0], p[4]
    like = dict(dtype=torch.int32, device=pool.device)
    if table_out is None:
        table_out = torch.empty((n, width), **like)
    if lens_out is None:
        lens_out = torch.empty(n, **like)
    if refs is None:
        refs = torch.empty(pages, **like)
    buf = (ws or Workspace(pool.device)).get(size(rows, n, width, pages))
    i32 = torch.int32
    rc = call(_POOL.set(*p)[0], _array(table, i32, pool, (rows, width), "table"),
              _array(lens, i32, pool, (rows,), "lens"), rows, width,
              _array(parent, i32, pool, (n,), "parent"),
              None if room is None else _array(room, i32, pool, (n,), "room"), n,
              _array(table_out, i32, pool, (n, width), "table_out"),
              _array(lens_out, i32, pool, (n,), "lens_out"),
              _array(refs, i32, pool, (pages,), "refs"), _ptr(diag), buf.data_ptr(), buf.numel(),
              _stream(stream, pool, buf, table_out, lens_out, refs))
    if rc:
        opattr._check(rc, "opattr_pages_fork")
    return Outputs(table=table_out, lens=lens_out, refs=refs)


def opattr_pages_compact(pool, table, held=None, table_out=None, moved=None, live=None,
                         ws: Workspace | None = None, diag=None, stream=None) -> Outputs:
    """The pages in use moved to the front of the pool. Returns the table with
    their new places, moved (each page's new place, -1: free) and live [1], how
    many are in use."""
    call, size = _entry("opattr_pages_compact"), _call["opattr_pages_compact_workspace_bytes"]
    if table.dim() != 2:
        raise ValueError("table is [rows, entries]")
    p = _pool(pool, 1, held)
    (rows, width), pages = table.shape, p[4]
    like = dict(dtype=torch.int32, device=pool.device)
    if table_out is None:
        table_out = torch.empty((rows, width), **like)
    if moved is None:
        moved = torch.empty(pages, **like)
    if live is None:
        live = torch.empty(1, **like)
    buf = (ws or Workspace(pool.device)).get(size(pages))
    i32 = torch.int32
    rc = call(_POOL.set(*p)[0], _array(table, i32, pool, (rows, width), "table"), rows, width,
              _array(table_out, i32, pool, (rows, width), "table_out"),
              _array(moved, i32, pool, (pages,), "moved"), _array(live, i32, pool, (1,), "live"),
              _ptr(diag), buf.data_ptr(), buf.numel(),
              _stream(stream, pool, buf, table_out, moved, live))
    if rc:
        opattr._check(rc, "opattr_pages_compact")
    return Outputs(table=table_out, moved=moved, live=live)
