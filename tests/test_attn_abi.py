"""Host-side checks of the attention operators' C ABI and binding (no GPU): the
header against the binding, workspace sizes, refusals; and the 64-bit oracle of
the GPU tests against differences and plain loops."""
import ctypes as C
import os
import re
import subprocess

import numpy as np
import pytest

import attn_oracle as O
from paper_2609_11938_amd import attn, opattr

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "opattr_attn.h")
FAKE = 0x10000  # never dereferenced on the host
INVALID, WORKSPACE = -1, -2


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(opattr.LIB_PATH):
        from paper_2609_11938_amd import build

        build.build()
    return attn.library()


def test_header_declares_the_expected_calls(lib):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    assert sorted(set(re.findall(r"\b(opattr_[a-z_]+)\s*\(", text))) == sorted(attn.EXPORTS)
    out = subprocess.run(["nm", "-D", "--defined-only", opattr.LIB_PATH], check=True,
                         capture_output=True, text=True).stdout
    exported = set(re.findall(r"\sT\s(opattr_\w+)", out))
    assert set(attn.EXPORTS) <= exported


def test_struct_layouts_match_header(tmp_path):
    structs = {c.__name__: c for c in (attn.opattr_rows, attn.opattr_attn_shape,
                                       attn.opattr_kv_pages, attn.opattr_page_pool)}
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "opattr_attn.h"',
             "int main(void) {"]
    for name, cls in structs.items():
        lines.append(f'  printf("{name} %zu\\n", sizeof({name}));')
        for f, _ in cls._fields_:
            lines.append(f'  printf("{name}.{f} %zu\\n", offsetof({name}, {f}));')
    lines += ["  return 0;", "}"]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines) + "\n")
    subprocess.run(["gcc", "-std=c11", "-I", os.path.dirname(HEADER), "-o", str(exe), str(src)],
                   check=True)
    got = dict(line.split() for line in subprocess.run([str(exe)], check=True, capture_output=True,
                                                       text=True).stdout.splitlines())
    for name, cls in structs.items():
        assert int(got[name]) == C.sizeof(cls), name
        for f, _ in cls._fields_:
            assert int(got[f"{name}.{f}"]) == getattr(cls, f).offset, f"{name}.{f}"


def _shape(**kw):
    a = dict(n_q=100, n_k=100, cu_q=FAKE, cu_k=FAKE, n_seqs=2, n_heads=8, n_kv_heads=2,
             head_dim=64, dtype=0, causal=1, scale=0.125)
    a.update(kw)
    return attn.opattr_attn_shape(**a)


def _rows(p=FAKE, ts=512, hs=64):
    return attn.opattr_rows(p, ts, hs)


BAD_SHAPES = [dict(n_q=-1), dict(n_k=-1), dict(n_q=1 << 30), dict(n_seqs=-1), dict(cu_q=None),
              dict(cu_k=None), dict(n_heads=0), dict(n_kv_heads=0), dict(n_heads=9),
              dict(head_dim=0), dict(head_dim=60), dict(head_dim=136), dict(dtype=2),
              dict(causal=2), dict(scale=float("nan")), dict(scale=float("inf"))]
BAD_ROWS = [None, dict(p=None), dict(p=FAKE + 2), dict(ts=56), dict(ts=516), dict(hs=-8),
            dict(hs=68), dict(ts=1 << 23)]


@pytest.mark.parametrize("bad", BAD_SHAPES, ids=str)
def test_prompt_refuses_shapes(lib, bad):
    r = _rows()
    a = _shape(**bad)
    assert lib.opattr_attn_prompt(a, r, r, r, r, FAKE, None, None) == INVALID
    assert lib.opattr_attn_prompt_grad_workspace_bytes(a) == 0
    assert lib.opattr_attn_prompt_grad(a, r, r, r, r, r, FAKE, r, r, r, None, FAKE, 1 << 30,
                                       None) == INVALID


@pytest.mark.parametrize("bad", BAD_ROWS, ids=str)
def test_prompt_refuses_rows(lib, bad):
    r, x = _rows(), None if bad is None else _rows(**bad)
    for at in range(4):
        rows = [r] * 4
        rows[at] = x
        assert lib.opattr_attn_prompt(_shape(), *rows, FAKE, None, None) == INVALID, at
    for at in (0, 1, 2, 3, 4, 6, 7, 8):
        args = [r, r, r, r, r, FAKE, r, r, r]
        args[at] = x
        assert lib.opattr_attn_prompt_grad(_shape(), *args, None, FAKE, 1 << 30, None) == INVALID
    assert lib.opattr_attn_prompt(None, r, r, r, r, FAKE, None, None) == INVALID


def test_grad_workspace_and_lse(lib):
    r, a = _rows(), _shape()
    need = lib.opattr_attn_prompt_grad_workspace_bytes(a)
    assert need >= 100 * 8 * 4
    for ws, n in ((None, need), (FAKE, need - 1), (FAKE + 16, need)):
        assert lib.opattr_attn_prompt_grad(a, r, r, r, r, r, FAKE, r, r, r, None, ws, n,
                                           None) == WORKSPACE
    assert lib.opattr_attn_prompt_grad(a, r, r, r, r, r, None, r, r, r, None, FAKE, need,
                                       None) == INVALID


def _pages(**kw):
    a = dict(k=FAKE, v=FAKE, page_stride=4096, token_stride=128, head_stride=64, n_pages=10,
             page_size=16, table=FAKE, n_seqs=3, table_stride=5, n_kv_heads=2, head_dim=64,
             dtype=0)
    a.update(kw)
    return attn.opattr_kv_pages(**a)


BAD_PAGES = [dict(k=None), dict(v=None), dict(k=FAKE + 4), dict(page_stride=4100),
             dict(token_stride=-8), dict(head_stride=4), dict(n_pages=-1), dict(page_size=0),
             dict(page_size=24), dict(page_size=2048), dict(table=None), dict(n_seqs=-1),
             dict(table_stride=-1), dict(table_stride=1 << 28), dict(n_kv_heads=0),
             dict(head_dim=4), dict(head_dim=256), dict(dtype=-1)]


@pytest.mark.parametrize("bad", BAD_PAGES, ids=str)
def test_paged_refuses_pages(lib, bad):
    r, c = _rows(), _pages(**bad)
    assert lib.opattr_attn_paged(c, 8, r, FAKE, 0.1, r, FAKE, None, FAKE, 1 << 30,
                                 None) == INVALID
    assert lib.opattr_kv_append(c, 3, FAKE, r, r, FAKE, None, None, None) == INVALID
    assert lib.opattr_attn_paged_workspace_bytes(c, 8) == 0


def test_paged_refuses(lib):
    r, c = _rows(), _pages(table_stride=500)
    call = lib.opattr_attn_paged
    for heads in (0, 3, 2 * 17):
        assert call(c, heads, r, FAKE, 0.1, r, FAKE, None, FAKE, 1 << 30, None) == INVALID
    assert call(c, 8, r, None, 0.1, r, FAKE, None, FAKE, 1 << 30, None) == INVALID
    assert call(c, 8, r, FAKE, float("nan"), r, FAKE, None, FAKE, 1 << 30, None) == INVALID
    assert call(c, 8, _rows(hs=3), FAKE, 0.1, r, FAKE, None, FAKE, 1 << 30, None) == INVALID
    assert call(c, 8, r, FAKE, 0.1, None, FAKE, None, FAKE, 1 << 30, None) == INVALID
    need = lib.opattr_attn_paged_workspace_bytes(c, 8)
    assert need > 0
    assert call(c, 8, r, FAKE, 0.1, r, FAKE, None, FAKE, need - 1, None) == WORKSPACE
    assert call(c, 8, r, FAKE, 0.1, r, FAKE, None, None, need, None) == WORKSPACE


def test_append_refuses(lib):
    r, c = _rows(), _pages()
    call = lib.opattr_kv_append
    assert call(c, -1, FAKE, r, r, FAKE, None, None, None) == INVALID
    assert call(c, 3, None, r, r, FAKE, None, None, None) == INVALID
    assert call(c, 3, FAKE, r, r, None, None, None, None) == INVALID
    assert call(c, 3, FAKE, _rows(p=None), r, FAKE, None, None, None) == INVALID
    assert call(c, 3, FAKE, r, None, FAKE, None, None, None) == INVALID
    assert call(c, 3, FAKE, r, r, FAKE, FAKE, None, None) == INVALID  # lens_out is lens
    assert call(None, 3, FAKE, r, r, FAKE, None, None, None) == INVALID


def _pool(**kw):
    a = dict(data=FAKE, plane_stride=1 << 20, page_stride=4096, n_planes=4, n_pages=100,
             page_bytes=4096, page_size=16, held=None)
    a.update(kw)
    return attn.opattr_page_pool(**a)


@pytest.mark.parametrize("bad", [dict(data=None), dict(data=FAKE + 8), dict(plane_stride=8),
                                 dict(page_stride=2048), dict(page_stride=4100),
                                 dict(n_planes=-1), dict(n_pages=-1), dict(n_pages=1 << 25),
                                 dict(page_bytes=100), dict(page_size=0)], ids=str)
def test_pages_refuse_pools(lib, bad):
    p = _pool(**bad)
    assert lib.opattr_pages_fork(p, FAKE, FAKE, 4, 5, FAKE, FAKE, 6, 2 * FAKE, 3 * FAKE, None,
                                 None, FAKE, 1 << 30, None) == INVALID
    assert lib.opattr_pages_compact(p, FAKE, 4, 5, 2 * FAKE, FAKE, None, None, FAKE, 1 << 30,
                                    None) == INVALID


def test_pages_refuse_tables(lib):
    p, big = _pool(), 1 << 30
    fork, compact = lib.opattr_pages_fork, lib.opattr_pages_compact
    for args in ((None, FAKE, 4, 5, FAKE, FAKE, 6, 2 * FAKE, 3 * FAKE),
                 (FAKE, None, 4, 5, FAKE, FAKE, 6, 2 * FAKE, 3 * FAKE),
                 (FAKE, FAKE, -1, 5, FAKE, FAKE, 6, 2 * FAKE, 3 * FAKE),
                 (FAKE, FAKE, 4, -1, FAKE, FAKE, 6, 2 * FAKE, 3 * FAKE),
                 (FAKE, FAKE, 4, 5, None, FAKE, 6, 2 * FAKE, 3 * FAKE),
                 (FAKE, FAKE, 4, 5, FAKE, FAKE, 6, None, 3 * FAKE),
                 (FAKE, FAKE, 4, 5, FAKE, FAKE, 6, FAKE, 3 * FAKE),
                 (FAKE, FAKE, 4, 5, FAKE, FAKE, 6, 2 * FAKE, FAKE),
                 (FAKE, FAKE, 4, 5, FAKE, FAKE, 6, 2 * FAKE, None)):
        assert fork(p, *args, None, None, FAKE, big, None) == INVALID, args
    need = lib.opattr_pages_fork_workspace_bytes(4, 6, 5, 100)
    assert fork(p, FAKE, FAKE, 4, 5, FAKE, FAKE, 6, 2 * FAKE, 3 * FAKE, None, None, FAKE,
                need - 1, None) == WORKSPACE
    assert lib.opattr_pages_fork_workspace_bytes(-1, 6, 5, 100) == 0
    assert compact(p, None, 4, 5, FAKE, FAKE, None, None, FAKE, big, None) == INVALID
    assert compact(p, FAKE, 4, 5, None, FAKE, None, None, FAKE, big, None) == INVALID
    assert compact(p, FAKE, 4, 5, FAKE, None, None, None, FAKE, big, None) == INVALID
    assert compact(p, FAKE, 1 << 20, 5, FAKE, FAKE, None, None, FAKE, big, None) == INVALID
    need = lib.opattr_pages_compact_workspace_bytes(100)
    assert compact(p, FAKE, 4, 5, FAKE, FAKE, None, None, FAKE, need - 1, None) == WORKSPACE
    assert lib.opattr_pages_compact_workspace_bytes(1 << 25) == 0


def test_binding_refuses_host_tensors(lib):
    import torch

    q = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    cu = torch.tensor([0, 4], dtype=torch.int32)
    with pytest.raises(TypeError):
        attn.opattr_attn_prompt(q, q, q, cu)


# --------------------------------------------------------------------------- #
# the oracle                                                                  #
# --------------------------------------------------------------------------- #


@pytest.mark.parametrize("n,m,causal", [(5, 5, True), (4, 9, True), (9, 4, True), (6, 3, False),
                                        (3, 0, False)])
def test_oracle_against_loops_and_differences(n, m, causal):
    rng = np.random.default_rng(n * 10 + m)
    d, scale = 8, 0.3
    q, k, v = rng.normal(size=(n, d)), rng.normal(size=(m, d)), rng.normal(size=(m, d))
    dout = rng.normal(size=(n, d))

    def loss(q, k, v):
        s = 0.0
        for i in range(n):
            js = [j for j in range(m) if not causal or j <= i + m - n]
            w = [np.exp(scale * q[i] @ k[j]) for j in js]
            for j, x in zip(js, w):
                s += x / sum(w) * (v[j] @ dout[i])
        return s

    got = O.head(q, k, v, scale, causal, "bfloat16", dout)
    assert abs((got["out"][0] * dout).sum() - loss(q, k, v)) < 1e-12
    for name, t in (("dq", q), ("dk", k), ("dv", v)):
        way = rng.normal(size=t.shape)
        h = 1e-5
        args = {"dq": q, "dk": k, "dv": v}
        up, down = dict(args), dict(args)
        up[name], down[name] = t + h * way, t - h * way
        diff = (loss(up["dq"], up["dk"], up["dv"]) - loss(down["dq"], down["dk"], down["dv"])) / \
            (2 * h)
        assert abs(diff - (got[name][0] * way).sum()) < 1e-7, name


def test_oracle_bounds_fail_a_wrong_result():
    """The bounds are narrow enough to catch a mistake: a key left out, a mask off
    by one, a wrong scale."""
    rng = np.random.default_rng(3)
    n, d = 40, 64
    q, k, v, dout = (rng.normal(size=(n, d)) for _ in range(4))
    good = O.head(q, k, v, 0.125, True, "bfloat16", dout)
    wrong = {"scale": O.head(q, k, v, 0.13, True, "bfloat16", dout),
             "mask": O.head(q, k, v, 0.125, False, "bfloat16", dout),
             "key": O.head(q[1:], k[1:], v[1:], 0.125, True, "bfloat16", dout[1:])}
    for what, bad in wrong.items():
        for name in ("out", "dq", "dk", "dv"):
            value, bound = good[name]
            value, bound = value[-len(bad[name][0]):], bound[-len(bad[name][0]):]
            assert (np.abs(bad[name][0] - value) > bound).any(), (what, name)


def test_calls_past_one_launch_are_refused(lib):
    """A launch takes fewer than 2^32 threads: what would need more is an
    argument error, found before anything is enqueued."""
    r = _rows()
    a = _shape(n_heads=64, n_kv_heads=64, n_seqs=1 << 19)
    assert lib.opattr_attn_prompt(a, r, r, r, r, FAKE, None, None) == INVALID
    assert lib.opattr_attn_prompt_grad_workspace_bytes(a) == 0
    c = _pages(n_seqs=1 << 19)
    assert lib.opattr_attn_paged(c, 32, r, FAKE, 0.1, r, FAKE, None, FAKE, 1 << 30,
                                 None) == INVALID
    assert lib.opattr_kv_append(_pages(), 1 << 27, FAKE, r, r, FAKE, None, None, None) == INVALID


OVERLAPS = [dict(hs=0), dict(hs=56), dict(ts=504), dict(ts=64, hs=64), dict(ts=128, hs=320),
            dict(ts=3584, hs=512)]


@pytest.mark.parametrize("bad", OVERLAPS, ids=str)
def test_outputs_that_overlap_themselves_are_refused(lib, bad):
    """8 heads of 64, 100 tokens: two rows of the output in one place."""
    r, x = _rows(), _rows(**bad)
    a = _shape(n_heads=8, n_kv_heads=8)
    assert lib.opattr_attn_prompt(a, r, r, r, x, FAKE, None, None) == INVALID
    for at in (6, 7, 8):
        args = [r, r, r, r, r, FAKE, r, r, r]
        args[at] = x
        assert lib.opattr_attn_prompt_grad(a, *args, None, FAKE, 1 << 40, None) == INVALID, at
    c = _pages(n_seqs=100, table_stride=1)
    assert lib.opattr_attn_paged(c, 8, r, FAKE, 0.1, x, FAKE, None, FAKE, 1 << 30,
                                 None) == INVALID


@pytest.mark.parametrize("good", [dict(), dict(hs=6400, ts=64), dict(ts=1024, hs=120),
                                  dict(ts=192, hs=64 * 3 * 100), dict(ts=128, hs=64 + 128 * 100),
                                  dict(ts=3200, hs=320)], ids=str)
def test_outputs_of_other_orders_pass(lib, good):
    """Heads before tokens, gaps, heads between tokens: taken (the call ends at its
    missing workspace)."""
    r, x = _rows(), _rows(**good)
    a = _shape(n_heads=8, n_kv_heads=8)
    args = [r, r, r, r, r, FAKE, x, x, x]
    assert lib.opattr_attn_prompt_grad(a, *args, None, None, 0, None) == WORKSPACE


def test_caches_and_pools_that_overlap_themselves_are_refused(lib):
    r = _rows()
    for bad in (dict(page_stride=0), dict(token_stride=0), dict(head_stride=0),
                dict(token_stride=64), dict(page_stride=2040), dict(page_stride=128 * 15)):
        assert lib.opattr_kv_append(_pages(**bad), 3, FAKE, r, r, FAKE, None, None,
                                    None) == INVALID, bad
    for bad in (dict(plane_stride=0), dict(plane_stride=4096 * 99), dict(plane_stride=2048)):
        p = _pool(**bad)
        assert lib.opattr_pages_fork(p, FAKE, FAKE, 4, 5, FAKE, FAKE, 6, 2 * FAKE, 3 * FAKE, None,
                                     None, FAKE, 1 << 30, None) == INVALID, bad
        assert lib.opattr_pages_compact(p, FAKE, 4, 5, 2 * FAKE, FAKE, None, None, FAKE, 1 << 30,
                                        None) == INVALID, bad
    # planes between the pages: taken (the call ends at its missing workspace)
    p = _pool(plane_stride=4096, page_stride=4 * 4096)
    assert lib.opattr_pages_compact(p, FAKE, 4, 5, 2 * FAKE, FAKE, None, None, None, 0,
                                    None) == WORKSPACE


def test_overlap_rule_against_places(lib):
    """The rule for every pair of strides of a small output, against its places."""
    r = _rows()
    n, heads, d = 5, 3, 16
    a = _shape(n_q=n, n_k=n, n_heads=heads, n_kv_heads=heads, head_dim=d)
    for ts in range(16, 96, 8):
        for hs in range(0, 136, 8):
            at = [t * ts + h * hs + e for t in range(n) for h in range(heads) for e in range(d)]
            x = _rows(ts=ts, hs=hs)
            want = INVALID if len(set(at)) < len(at) else WORKSPACE
            assert lib.opattr_attn_prompt_grad(a, r, r, r, r, r, FAKE, x, x, x, None, None, 0,
                                               None) == want, (ts, hs)


def test_overlap_rule_of_caches_against_places(lib):
    """So for caches, of which the overlapping ones only: the others would go on."""
    r = _rows()
    pages, size, heads, d = 3, 2, 3, 8
    for ps in range(0, 120, 8):
        for ts in range(0, 72, 8):
            for hs in range(0, 72, 8):
                at = [x * ps + t * ts + h * hs + e for x in range(pages) for t in range(size)
                      for h in range(heads) for e in range(d)]
                if len(set(at)) == len(at):
                    continue
                c = _pages(n_pages=pages, page_size=size, n_kv_heads=heads, head_dim=d,
                           page_stride=ps, token_stride=ts, head_stride=hs)
                assert lib.opattr_kv_append(c, 3, FAKE, r, r, FAKE, None, None,
                                            None) == INVALID, (ps, ts, hs)


def test_counts_written_where_they_are_read_are_refused(lib):
    """Every block reads held while the first ones to be done write refs or moved."""
    p, big = _pool(held=5 * FAKE), 1 << 30
    assert lib.opattr_pages_fork(p, FAKE, FAKE, 4, 5, FAKE, FAKE, 6, 2 * FAKE, 3 * FAKE, 5 * FAKE,
                                 None, FAKE, big, None) == INVALID
    assert lib.opattr_pages_compact(p, FAKE, 4, 5, 2 * FAKE, 5 * FAKE, None, None, FAKE, big,
                                    None) == INVALID
