"""Python binding of the attention operators of libopattr (include/opattr_attn.h).

Argument marshalling only, as in ``opattr``: torch device tensors are handed to
the C entry points by pointer, outputs are written where the caller says (or
into new tensors), and the work goes to the current HIP stream. There is no CPU
fallback: a missing library raises.

Tensors of queries, keys, values, outputs and gradients are [tokens, heads,
head_dim] in bfloat16 or float16, any strides with the last one 1 (multiples of
8 elements, 16-byte aligned). Lengths, offsets and page tables are contiguous
int32 tensors. Data errors go to the ``diag`` record, if one is given
(``new_diag``; read it with ``opattr.read_diag``). A ``Workspace`` serves one
call at a time: calls that may overlap on two streams need one each. Autograd does not see the
calls: with it on, queries, keys and values that require a gradient are refused;
``opattr_attn_prompt_grad`` takes them and is the gradient.
"""
from __future__ import annotations

import ctypes as C
import importlib.util
import os

import torch

from . import opattr
from .opattr import Outputs, Workspace  # noqa: F401  (part of this interface)

BF16, F16 = 0, 1  # OPATTR_BF16, OPATTR_F16


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


class opattr_kv_scaled(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("page_stride", C.c_int64),
                ("token_stride", C.c_int64), ("head_stride", C.c_int64), ("k_scale", C.c_void_p),
                ("v_scale", C.c_void_p), ("scale_page_stride", C.c_int64),
                ("scale_block_stride", C.c_int64), ("scale_head_stride", C.c_int64),
                ("n_pages", C.c_int32), ("page_size", C.c_int32), ("block_size", C.c_int32),
                ("table", C.c_void_p), ("n_seqs", C.c_int32), ("table_stride", C.c_int32),
                ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("dtype", C.c_int32)]


class opattr_page_pool(C.Structure):
    _fields_ = [("data", C.c_void_p), ("plane_stride", C.c_int64), ("page_stride", C.c_int64),
                ("n_planes", C.c_int32), ("n_pages", C.c_int32), ("page_bytes", C.c_int32),
                ("page_size", C.c_int32), ("held", C.c_void_p)]


EXPORTS = ("opattr_attn_prompt", "opattr_attn_prompt_grad",
           "opattr_attn_prompt_grad_workspace_bytes", "opattr_attn_paged",
           "opattr_attn_paged_workspace_bytes", "opattr_kv_append",
           "opattr_attn_prompt_window", "opattr_attn_prompt_window_grad",
           "opattr_attn_prompt_window_grad_workspace_bytes", "opattr_attn_paged_window",
           "opattr_attn_paged_window_workspace_bytes", "opattr_kv_append_scaled",
           "opattr_attn_paged_scaled", "opattr_attn_paged_scaled_workspace_bytes",
           "opattr_pages_fork",
           "opattr_pages_fork_workspace_bytes", "opattr_pages_compact",
           "opattr_pages_compact_workspace_bytes")

BIND_PATH = os.path.join(os.path.dirname(opattr.LIB_PATH), "attn_bind.so")

_lib = None
_bind = None


def library():
    """libopattr with the attention entry points declared (for callers of the C
    ABI; the functions below go through ``binding``)."""
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
    L.opattr_attn_prompt_window.argtypes = [P(opattr_attn_shape), i32, i32, rows, rows, rows, rows,
                                            vp, vp, vp]
    L.opattr_attn_prompt_window_grad_workspace_bytes.argtypes = [P(opattr_attn_shape), i32, i32]
    L.opattr_attn_prompt_window_grad.argtypes = [P(opattr_attn_shape), i32, i32, rows, rows, rows,
                                                 rows, rows, vp, rows, rows, rows, vp, vp, sz, vp]
    L.opattr_attn_paged_window_workspace_bytes.argtypes = [P(opattr_kv_pages), i32, i32, i32]
    L.opattr_attn_paged_window.argtypes = [P(opattr_kv_pages), i32, i32, i32, rows, vp, C.c_float,
                                           rows, vp, vp, vp, sz, vp]
    L.opattr_kv_append_scaled.argtypes = [P(opattr_kv_scaled), i64, vp, rows, rows, vp, vp, vp, vp]
    L.opattr_attn_paged_scaled_workspace_bytes.argtypes = [P(opattr_kv_scaled), i32, i32, i32]
    L.opattr_attn_paged_scaled.argtypes = [P(opattr_kv_scaled), i32, i32, i32, rows, vp, C.c_float,
                                           rows, vp, vp, vp, sz, vp]
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


def binding():
    """The compiled marshalling (csrc/attn_bind.cpp). Raises when it is not
    built."""
    global _bind
    if _bind is None:
        if not os.path.exists(BIND_PATH):
            raise RuntimeError(f"attn_bind is not built ({BIND_PATH}); run "
                               "__graft_entry__.build()")
        opattr.library()
        spec = importlib.util.spec_from_file_location("attn_bind", BIND_PATH)
        _bind = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(_bind)
    return _bind


def new_diag(device="cuda:0", stream=None):
    """A cleared diag record on the device, of the stream's own memory (None: the
    device's current stream)."""
    before = torch.cuda.current_stream(device)
    if stream is None:
        stream = before
    with torch.cuda.stream(stream):
        diag = opattr._new_diag(device, stream)
    diag.record_stream(before)
    return diag


def _on(stream, call, *args, ws=None, **kw):
    """The call with ``stream`` as the current one, so that what it allocates is
    that stream's own: memory that the present stream still works on is not given
    out. The memory of every tensor it uses is kept until the stream has passed
    the call, that of its results also for the present stream."""
    before = torch.cuda.current_stream(stream.device)
    with torch.cuda.stream(stream):
        if ws is not None:
            kw["ws"] = ws
        result = call(*args, **kw)
    made = [result] if torch.is_tensor(result) else \
        list(result.values() if isinstance(result, dict) else result)
    for t in (*args, *kw.values(), *made):
        if torch.is_tensor(t):
            t.record_stream(stream)
    for t in made:
        t.record_stream(before)
    return result


def _with_workspace(call, ws, device, before, diag):
    """call(*before, workspace, diag), with as large a workspace as it asks for."""
    need = call(*before, None if ws is None else ws.buf, diag)
    if need is not None:
        call(*before, (ws or Workspace(device)).get(need), diag)


def opattr_attn_prompt(q, k, v, cu_q, cu_k=None, causal=True, scale=None, out=None, lse=None,
                       diag=None, stream=None):
    """Attention over packed prompts: (out, lse). Sequence b has queries
    q[cu_q[b]:cu_q[b+1]] and keys k[cu_k[b]:cu_k[b+1]] (cu_k None: as cu_q);
    scale None: 1 / sqrt(head_dim). Rows of ``out`` and ``lse`` outside every
    sequence are not written."""
    if stream is not None:
        return _on(stream, opattr_attn_prompt, q, k, v, cu_q, cu_k, causal,
                   scale, out, lse, diag=diag)
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    if lse is None:
        lse = torch.empty(q.shape[1::-1], dtype=torch.float32, device=q.device)
    (_bind or binding()).attn_prompt(q, k, v, cu_q, cu_k, causal, scale, out, lse, diag)
    return out, lse


def opattr_attn_prompt_grad(dout, q, k, v, out, lse, cu_q, cu_k=None, causal=True, scale=None,
                            dq=None, dk=None, dv=None, ws: Workspace | None = None, diag=None,
                            stream=None):
    """Gradients of sum(out * dout): (dq, dk, dv). out and lse are
    opattr_attn_prompt's for the same inputs."""
    if stream is not None:
        return _on(stream, opattr_attn_prompt_grad, dout, q, k, v, out, lse,
                   cu_q, cu_k, causal, scale, dq, dk, dv, ws=ws, diag=diag)
    if dq is None:
        dq = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    if dk is None:
        dk = torch.empty(k.shape, dtype=q.dtype, device=q.device)
    if dv is None:
        dv = torch.empty(k.shape, dtype=q.dtype, device=q.device)
    _with_workspace((_bind or binding()).attn_prompt_grad, ws, q.device,
                    (dout, q, k, v, out, lse, cu_q, cu_k, causal, scale, dq, dk, dv), diag)
    return dq, dk, dv


def opattr_attn_paged(q, k_pages, v_pages, table, lens, scale=None, out=None, lse=None,
                      ws: Workspace | None = None, diag=None, stream=None):
    """Attention of one token a sequence, q [sequences, heads, head_dim], over
    the first lens[b] tokens of each: (out, lse [heads, sequences])."""
    if stream is not None:
        return _on(stream, opattr_attn_paged, q, k_pages, v_pages, table, lens,
                   scale, out, lse, ws=ws, diag=diag)
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    if lse is None:
        lse = torch.empty(q.shape[1::-1], dtype=torch.float32, device=q.device)
    _with_workspace((_bind or binding()).attn_paged, ws, q.device,
                    (q, k_pages, v_pages, table, lens, scale, out, lse), diag)
    return out, lse


def opattr_kv_append(k_new, v_new, cu, k_pages, v_pages, table, lens, lens_out=None, diag=None,
                     stream=None):
    """Rows cu[b] .. cu[b+1] of k_new and v_new become the next tokens of
    sequence b, which holds lens[b]; returns the new lengths."""
    if stream is not None:
        return _on(stream, opattr_kv_append, k_new, v_new, cu, k_pages, v_pages,
                   table, lens, lens_out, diag=diag)
    if lens_out is None:
        lens_out = torch.empty(lens.shape, dtype=torch.int32, device=k_pages.device)
    (_bind or binding()).kv_append(k_new, v_new, cu, k_pages, v_pages, table, lens, lens_out,
                                   diag)
    return lens_out


def opattr_attn_prompt_window(q, k, v, cu_q, window, sinks=0, cu_k=None, scale=None, out=None,
                              lse=None, diag=None, stream=None):
    """Causal attention over packed prompts through a sliding window: (out, lse). A
    query sees the last ``window`` keys up to its own place, and the first ``sinks``
    of its sequence; the rest as in opattr_attn_prompt."""
    if stream is not None:
        return _on(stream, opattr_attn_prompt_window, q, k, v, cu_q, window, sinks, cu_k, scale,
                   out, lse, diag=diag)
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    if lse is None:
        lse = torch.empty(q.shape[1::-1], dtype=torch.float32, device=q.device)
    (_bind or binding()).attn_prompt_window(q, k, v, cu_q, cu_k, window, sinks, scale, out, lse,
                                            diag)
    return out, lse


def opattr_attn_prompt_window_grad(dout, q, k, v, out, lse, cu_q, window, sinks=0, cu_k=None,
                                   scale=None, dq=None, dk=None, dv=None,
                                   ws: Workspace | None = None, diag=None, stream=None):
    """Gradients of sum(out * dout): (dq, dk, dv). out and lse are
    opattr_attn_prompt_window's for the same inputs."""
    if stream is not None:
        return _on(stream, opattr_attn_prompt_window_grad, dout, q, k, v, out, lse, cu_q, window,
                   sinks, cu_k, scale, dq, dk, dv, ws=ws, diag=diag)
    if dq is None:
        dq = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    if dk is None:
        dk = torch.empty(k.shape, dtype=q.dtype, device=q.device)
    if dv is None:
        dv = torch.empty(k.shape, dtype=q.dtype, device=q.device)
    _with_workspace((_bind or binding()).attn_prompt_window_grad, ws, q.device,
                    (dout, q, k, v, out, lse, cu_q, cu_k, window, sinks, scale, dq, dk, dv), diag)
    return dq, dk, dv


def opattr_attn_paged_window(q, k_pages, v_pages, table, lens, window, sinks=0, scale=None,
                             out=None, lse=None, ws: Workspace | None = None, diag=None,
                             stream=None):
    """Attention of one token a sequence over the last ``window`` and the first
    ``sinks`` of its lens[b] tokens: (out, lse [heads, sequences]). Pages of which no
    token is seen are not looked up."""
    if stream is not None:
        return _on(stream, opattr_attn_paged_window, q, k_pages, v_pages, table, lens, window,
                   sinks, scale, out, lse, ws=ws, diag=diag)
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    if lse is None:
        lse = torch.empty(q.shape[1::-1], dtype=torch.float32, device=q.device)
    _with_workspace((_bind or binding()).attn_paged_window, ws, q.device,
                    (q, k_pages, v_pages, table, lens, window, sinks, scale, out, lse), diag)
    return out, lse


def opattr_kv_append_scaled(k_new, v_new, cu, k_pages, v_pages, k_scales, v_scales, table, lens,
                            lens_out=None, diag=None, stream=None):
    """opattr_kv_append into a cache of 8 bits: codes k_pages and v_pages [pages,
    page_size, kv_heads, head_dim] (float8_e4m3fn or uint8), and an exponent's byte for
    each block of tokens and head, k_scales and v_scales [pages, blocks, kv_heads]
    (float8_e8m0fnu or uint8): page_size / blocks tokens a block. A block's exponent
    grows with its tokens, and what it holds is rounded to it again. Returns the new
    lengths."""
    if stream is not None:
        return _on(stream, opattr_kv_append_scaled, k_new, v_new, cu, k_pages, v_pages, k_scales,
                   v_scales, table, lens, lens_out, diag=diag)
    if lens_out is None:
        lens_out = torch.empty(lens.shape, dtype=torch.int32, device=k_pages.device)
    (_bind or binding()).kv_append_scaled(k_new, v_new, cu, k_pages, v_pages, k_scales, v_scales,
                                          table, lens, lens_out, diag)
    return lens_out


def opattr_attn_paged_scaled(q, k_pages, v_pages, k_scales, v_scales, table, lens, window=None,
                             sinks=0, scale=None, out=None, lse=None,
                             ws: Workspace | None = None, diag=None, stream=None):
    """Attention of one token a sequence over a cache of 8 bits (see
    opattr_kv_append_scaled): (out, lse [heads, sequences]). window None: all of the
    lens[b] tokens; else the last ``window`` and the first ``sinks``."""
    if stream is not None:
        return _on(stream, opattr_attn_paged_scaled, q, k_pages, v_pages, k_scales, v_scales,
                   table, lens, window, sinks, scale, out, lse, ws=ws, diag=diag)
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    if lse is None:
        lse = torch.empty(q.shape[1::-1], dtype=torch.float32, device=q.device)
    _with_workspace((_bind or binding()).attn_paged_scaled, ws, q.device,
                    (q, k_pages, v_pages, k_scales, v_scales, table, lens, window, sinks, scale,
                     out, lse), diag)
    return out, lse


def opattr_pages_fork(pool, page_size, table, lens, parent, room=None, held=None, table_out=None,
                      lens_out=None, refs=None, ws: Workspace | None = None, diag=None,
                      stream=None) -> Outputs:
    """The next page table: row i continues row parent[i] (-1: empty), with room
    for room[i] tokens. pool [planes, pages, ...] holds the pages that a forked
    row's last, part-filled page is copied in. Returns table, lens and refs."""
    if stream is not None:
        return _on(stream, opattr_pages_fork, pool, page_size, table, lens,
                   parent, room, held, table_out, lens_out, refs, ws=ws, diag=diag)
    like = dict(dtype=torch.int32, device=pool.device)
    if table_out is None:
        table_out = torch.empty((parent.shape[0], table.shape[1]), **like)
    if lens_out is None:
        lens_out = torch.empty(parent.shape, **like)
    if refs is None:
        refs = torch.empty(pool.shape[1], **like)
    _with_workspace((_bind or binding()).pages_fork, ws, pool.device,
                    (pool, page_size, table, lens, parent, room, held, table_out, lens_out,
                     refs), diag)
    return Outputs(table=table_out, lens=lens_out, refs=refs)


def opattr_pages_compact(pool, table, held=None, table_out=None, moved=None, live=None,
                         ws: Workspace | None = None, diag=None, stream=None) -> Outputs:
    """The pages in use moved to the front of the pool. Returns the table with
    their new places, moved (each page's new place, -1: free) and live [1], how
    many are in use."""
    if stream is not None:
        return _on(stream, opattr_pages_compact, pool, table, held, table_out,
                   moved, live, ws=ws, diag=diag)
    like = dict(dtype=torch.int32, device=pool.device)
    if table_out is None:
        table_out = torch.empty(table.shape, **like)
    if moved is None:
        moved = torch.empty(pool.shape[1], **like)
    if live is None:
        live = torch.empty(1, **like)
    _with_workspace((_bind or binding()).pages_compact, ws, pool.device,
                    (pool, table, held, table_out, moved, live), diag)
    return Outputs(table=table_out, moved=moved, live=live)
