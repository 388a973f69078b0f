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
    _lib = L
    return L


def new_diag(device="cuda:0", stream=None):
    """A cleared diag record on the device."""
    return opattr._new_diag(device, stream)


def _dtype(t):
    import torch

    if not t.is_cuda:
        raise TypeError("device tensors are taken")
    if t.dtype is torch.bfloat16:
        return BF16
    if t.dtype is torch.float16:
        return F16
    raise TypeError(f"bfloat16 or float16 tensors are taken, not {t.dtype}")


def _rows(t, like, tokens, heads, name):
    """The opattr_rows of a [tokens, heads, head_dim] tensor of like's type."""
    if t.dtype is not like.dtype or t.device != like.device:
        raise TypeError(f"{name}: {t.dtype} on {t.device}, expected {like.dtype} on {like.device}")
    d = like.shape[2]
    if t.shape != (tokens, heads, d):
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {(tokens, heads, d)}")
    ts, hs, es = t.stride()
    if es != 1 and d > 1:
        raise ValueError(f"{name}: the last dimension's values must lie side by side")
    if tokens <= 1:  # the stride of one row says nothing
        ts = d
    if heads == 1:
        hs = 0
    return opattr_rows(t.data_ptr(), ts, hs)


def _int32(t, n, like, name):
    import torch

    if t.dtype is not torch.int32 or t.device != like.device or not t.is_contiguous():
        raise TypeError(f"{name}: a contiguous int32 tensor on {like.device} is wanted")
    if n is not None and t.shape != (n if isinstance(n, tuple) else (n,)):
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {n}")
    return t.data_ptr()


def _float32(t, shape, like, name):
    import torch

    if t.dtype is not torch.float32 or t.device != like.device or not t.is_contiguous():
        raise TypeError(f"{name}: a contiguous float32 tensor on {like.device} is wanted")
    if t.shape != shape:
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {shape}")
    return t.data_ptr()


def _shape(q, k, cu_q, cu_k, causal, scale):
    if q.dim() != 3 or k.dim() != 3:
        raise ValueError("queries and keys are [tokens, heads, head_dim]")
    n = cu_q.shape[0] - 1
    if scale is None:
        scale = 1.0 / math.sqrt(q.shape[2])
    p = _int32(cu_q, None, q, "cu_q")
    return opattr_attn_shape(q.shape[0], k.shape[0], p,
                             p if cu_k is cu_q else _int32(cu_k, n + 1, q, "cu_k"), n,
                             q.shape[1], k.shape[1], q.shape[2], _dtype(q), 1 if causal else 0,
                             scale)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream(stream, *made):
    """The stream's handle. Tensors that a call made itself belong to the
    current stream: one used on another is kept until that has passed the call."""
    import torch

    if stream is None:
        return torch.cuda.current_stream().cuda_stream
    for t in made:
        t.record_stream(stream)
    return stream.cuda_stream


def opattr_attn_prompt(q, k, v, cu_q, cu_k=None, causal=True, scale=None, out=None, lse=None,
                       diag=None, stream=None):
    """Attention over packed prompts: (out, lse). Sequence b has queries
    q[cu_q[b]:cu_q[b+1]] and keys k[cu_k[b]:cu_k[b+1]] (cu_k None: as cu_q);
    scale None: 1 / sqrt(head_dim). Rows of ``out`` and ``lse`` outside every
    sequence are not written."""
    import torch

    L = library()
    cu_k = cu_q if cu_k is None else cu_k
    a = _shape(q, k, cu_q, cu_k, causal, scale)
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    if lse is None:
        lse = torch.empty((a.n_heads, a.n_q), dtype=torch.float32, device=q.device)
    rc = L.opattr_attn_prompt(
        a, _rows(q, q, a.n_q, a.n_heads, "q"), _rows(k, q, a.n_k, a.n_kv_heads, "k"),
        _rows(v, q, a.n_k, a.n_kv_heads, "v"), _rows(out, q, a.n_q, a.n_heads, "out"),
        _float32(lse, (a.n_heads, a.n_q), q, "lse"), _ptr(diag),
        _stream(stream, out, lse))
    opattr._check(rc, "opattr_attn_prompt")
    return out, lse


def opattr_attn_prompt_grad(dout, q, k, v, out, lse, cu_q, cu_k=None, causal=True, scale=None,
                            dq=None, dk=None, dv=None, ws: Workspace | None = None, diag=None,
                            stream=None):
    """Gradients of sum(out * dout): (dq, dk, dv). out and lse are
    opattr_attn_prompt's for the same inputs."""
    import torch

    L = library()
    cu_k = cu_q if cu_k is None else cu_k
    a = _shape(q, k, cu_q, cu_k, causal, scale)
    new = [torch.empty(t.shape, dtype=t.dtype, device=t.device) if g is None else g
           for g, t in ((dq, q), (dk, k), (dv, v))]
    need = L.opattr_attn_prompt_grad_workspace_bytes(a)
    buf = (ws or Workspace(q.device)).get(need)
    rc = L.opattr_attn_prompt_grad(
        a, _rows(dout, q, a.n_q, a.n_heads, "dout"), _rows(q, q, a.n_q, a.n_heads, "q"),
        _rows(k, q, a.n_k, a.n_kv_heads, "k"), _rows(v, q, a.n_k, a.n_kv_heads, "v"),
        _rows(out, q, a.n_q, a.n_heads, "out"), _float32(lse, (a.n_heads, a.n_q), q, "lse"),
        _rows(new[0], q, a.n_q, a.n_heads, "dq"), _rows(new[1], q, a.n_k, a.n_kv_heads, "dk"),
        _rows(new[2], q, a.n_k, a.n_kv_heads, "dv"), _ptr(diag), buf.data_ptr(), buf.numel(),
        _stream(stream, buf, *new))
    opattr._check(rc, "opattr_attn_prompt_grad")
    return tuple(new)


def _kv_pages(k_pages, v_pages, table):
    if k_pages.dim() != 4 or k_pages.shape != v_pages.shape or \
            k_pages.stride() != v_pages.stride() or k_pages.dtype is not v_pages.dtype:
        raise ValueError("k_pages and v_pages are [pages, page_size, kv_heads, head_dim], alike "
                         "in shape, strides and type")
    n, size, heads, d = k_pages.shape
    ps, ts, hs, es = k_pages.stride()
    if es != 1 and d > 1:
        raise ValueError("k_pages: the last dimension's values must lie side by side")
    if table.dim() != 2:
        raise ValueError("table is [sequences, entries]")
    return opattr_kv_pages(k_pages.data_ptr(), v_pages.data_ptr(), ps if n > 1 else 0,
                           ts if size > 1 else 0, hs if heads > 1 else 0, n, size,
                           _int32(table, None, k_pages, "table"), table.shape[0], table.shape[1],
                           heads, d, _dtype(k_pages))


def opattr_attn_paged(q, k_pages, v_pages, table, lens, scale=None, out=None, lse=None,
                      ws: Workspace | None = None, diag=None, stream=None):
    """Attention of one token a sequence, q [sequences, heads, head_dim], over
    the first lens[b] tokens of each: (out, lse [heads, sequences])."""
    import torch

    L = library()
    c = _kv_pages(k_pages, v_pages, table)
    b, h = c.n_seqs, q.shape[1]
    if scale is None:
        scale = 1.0 / math.sqrt(q.shape[2])
    if q.dtype is not k_pages.dtype or q.shape[2] != c.head_dim:
        raise ValueError("q: not of the cache's type and head_dim")
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    if lse is None:
        lse = torch.empty((h, b), dtype=torch.float32, device=q.device)
    buf = (ws or Workspace(q.device)).get(L.opattr_attn_paged_workspace_bytes(c, h))
    rc = L.opattr_attn_paged(c, h, _rows(q, q, b, h, "q"), _int32(lens, b, q, "lens"), scale,
                             _rows(out, q, b, h, "out"), _float32(lse, (h, b), q, "lse"),
                             _ptr(diag), buf.data_ptr(), buf.numel(),
                             _stream(stream, buf, out, lse))
    opattr._check(rc, "opattr_attn_paged")
    return out, lse


def opattr_kv_append(k_new, v_new, cu, k_pages, v_pages, table, lens, lens_out=None, diag=None,
                     stream=None):
    """Rows cu[b] .. cu[b+1] of k_new and v_new become the next tokens of
    sequence b, which holds lens[b]; returns the new lengths."""
    import torch

    L = library()
    c = _kv_pages(k_pages, v_pages, table)
    n, b = k_new.shape[0], c.n_seqs
    if k_new.dtype is not k_pages.dtype or k_new.shape[2] != c.head_dim:
        raise ValueError("k_new: not of the cache's type and head_dim")
    if lens_out is None:
        lens_out = torch.empty(b, dtype=torch.int32, device=k_pages.device)
    rc = L.opattr_kv_append(c, n, _int32(cu, b + 1, k_pages, "cu"),
                            _rows(k_new, k_new, n, c.n_kv_heads, "k_new"),
                            _rows(v_new, k_new, n, c.n_kv_heads, "v_new"),
                            _int32(lens, b, k_pages, "lens"),
                            _int32(lens_out, b, k_pages, "lens_out"), _ptr(diag),
                            _stream(stream, lens_out))
    opattr._check(rc, "opattr_kv_append")
    return lens_out


def _pool(pool, page_size, held):
    """The opattr_page_pool of a [planes, pages, ...] tensor whose pages lie in
    one piece each."""
    if pool.dim() < 3:
        raise ValueError("pool is [planes, pages, ...]")
    each = math.prod(pool.shape[2:])
    inner = 1
    for n, s in zip(reversed(pool.shape[2:]), reversed(pool.stride()[2:])):
        if n > 1 and s != inner:
            raise ValueError("a page's values must lie side by side")
        inner *= n
    size = pool.element_size()
    planes, pages = pool.shape[:2]
    return opattr_page_pool(pool.data_ptr(), pool.stride(0) * size if planes > 1 else 0,
                            pool.stride(1) * size if pages > 1 else each * size, planes, pages,
                            each * size, page_size,
                            None if held is None else _int32(held, pages, pool, "held"))


def opattr_pages_fork(pool, page_size, table, lens, parent, room=None, held=None, table_out=None,
                      lens_out=None, refs=None, ws: Workspace | None = None, diag=None,
                      stream=None) -> Outputs:
    """The next page table: row i continues row parent[i] (-1: empty), with room
    for room[i] tokens. pool [planes, pages, ...] holds the pages that a forked
    row's last, part-filled page is copied in. Returns table, lens and refs."""
    import torch

    L = library()
    if table.dim() != 2:
        raise ValueError("table is [rows, entries]")
    p = _pool(pool, page_size, held)
    rows, width, n = table.shape[0], table.shape[1], parent.shape[0]
    like = dict(dtype=torch.int32, device=pool.device)
    table_out = torch.empty((n, width), **like) if table_out is None else table_out
    lens_out = torch.empty(n, **like) if lens_out is None else lens_out
    refs = torch.empty(p.n_pages, **like) if refs is None else refs
    buf = (ws or Workspace(pool.device)).get(
        L.opattr_pages_fork_workspace_bytes(rows, n, width, p.n_pages))
    rc = L.opattr_pages_fork(
        p, _int32(table, None, pool, "table"), _int32(lens, rows, pool, "lens"), rows, width,
        _int32(parent, n, pool, "parent"),
        None if room is None else _int32(room, n, pool, "room"), n,
        _int32(table_out, (n, width), pool, "table_out"), _int32(lens_out, n, pool, "lens_out"),
        _int32(refs, p.n_pages, pool, "refs"), _ptr(diag), buf.data_ptr(), buf.numel(),
        _stream(stream, buf, table_out, lens_out, refs))
    opattr._check(rc, "opattr_pages_fork")
    return Outputs(table=table_out, lens=lens_out, refs=refs)


def opattr_pages_compact(pool, table, held=None, table_out=None, moved=None, live=None,
                         ws: Workspace | None = None, diag=None, stream=None) -> Outputs:
    """The pages in use moved to the front of the pool. Returns the table with
    their new places, moved (each page's new place, -1: free) and live [1], how
    many are in use."""
    import torch

    L = library()
    if table.dim() != 2:
        raise ValueError("table is [rows, entries]")
    p = _pool(pool, 1, held)
    like = dict(dtype=torch.int32, device=pool.device)
    table_out = torch.empty(table.shape, **like) if table_out is None else table_out
    moved = torch.empty(p.n_pages, **like) if moved is None else moved
    live = torch.empty(1, **like) if live is None else live
    buf = (ws or Workspace(pool.device)).get(L.opattr_pages_compact_workspace_bytes(p.n_pages))
    rc = L.opattr_pages_compact(p, _int32(table, None, pool, "table"), table.shape[0],
                                table.shape[1],
                                _int32(table_out, tuple(table.shape), pool, "table_out"),
                                _int32(moved, p.n_pages, pool, "moved"),
                                _int32(live, 1, pool, "live"), _ptr(diag), buf.data_ptr(),
                                buf.numel(),
                                _stream(stream, buf, table_out, moved, live))
    opattr._check(rc, "opattr_pages_compact")
    return Outputs(table=table_out, moved=moved, live=live)
