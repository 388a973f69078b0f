"""Host-side checks of window attention and of the paged cache of 8 bits (no GPU): the
header's struct against the binding, workspace sizes, refusals; and the 64-bit oracle
of the GPU tests against plain loops, differences and torch's e4m3."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest

import attn_window_oracle as W
from paper_2609_11938_amd import attn
from test_attn_abi import (BAD_PAGES, BAD_ROWS, BAD_SHAPES, FAKE, HEADER, INVALID, OVERLAPS,
                           WORKSPACE, _pages, _rows, _shape, lib)  # noqa: F401 (a fixture)

BIG = 1 << 30
BAD_WINDOWS = [(0, 0), (-1, 0), (-BIG, 5), (1, -1), (100, -BIG)]


def _prompt(lib, a, w, rows):  # noqa: F811
    return lib.opattr_attn_prompt_window(a, *w, *rows, FAKE, None, None)


def _grad(lib, a, w, rows, lse=FAKE, ws=FAKE, n=1 << 40):  # noqa: F811
    return lib.opattr_attn_prompt_window_grad(a, *w, *rows[:5], lse, *rows[5:], None, ws, n, None)


@pytest.mark.parametrize("bad", BAD_SHAPES + [dict(causal=0)], ids=str)
def test_window_refuses_shapes(lib, bad):  # noqa: F811
    a, r = _shape(**bad), _rows()
    assert _prompt(lib, a, (5, 1), [r] * 4) == INVALID
    assert lib.opattr_attn_prompt_window_grad_workspace_bytes(a, 5, 1) == 0
    assert _grad(lib, a, (5, 1), [r] * 8) == INVALID


@pytest.mark.parametrize("bad", BAD_WINDOWS, ids=str)
def test_bad_windows_are_refused(lib, bad):  # noqa: F811
    a, r, c = _shape(), _rows(), _pages()
    assert _prompt(lib, a, bad, [r] * 4) == INVALID
    assert lib.opattr_attn_prompt_window_grad_workspace_bytes(a, *bad) == 0
    assert _grad(lib, a, bad, [r] * 8) == INVALID
    assert lib.opattr_attn_paged_window(c, 8, *bad, r, FAKE, 0.1, r, FAKE, None, FAKE, BIG,
                                        None) == INVALID
    assert lib.opattr_attn_paged_window_workspace_bytes(c, 8, *bad) == 0
    c = _scaled()
    assert lib.opattr_attn_paged_scaled(c, 8, *bad, r, FAKE, 0.1, r, FAKE, None, FAKE, BIG,
                                        None) == INVALID
    assert lib.opattr_attn_paged_scaled_workspace_bytes(c, 8, *bad) == 0


@pytest.mark.parametrize("bad", BAD_ROWS, ids=str)
def test_window_refuses_rows(lib, bad):  # noqa: F811
    r, x = _rows(), None if bad is None else _rows(**bad)
    for at in range(4):
        rows = [r] * 4
        rows[at] = x
        assert _prompt(lib, _shape(), (5, 1), rows) == INVALID, at
    for at in range(8):
        rows = [r] * 8
        rows[at] = x
        assert _grad(lib, _shape(), (5, 1), rows) == INVALID, at
    assert _prompt(lib, None, (5, 1), [r] * 4) == INVALID
    assert _grad(lib, None, (5, 1), [r] * 8) == INVALID


@pytest.mark.parametrize("bad", OVERLAPS, ids=str)
def test_window_outputs_that_overlap_themselves_are_refused(lib, bad):  # noqa: F811
    r, x = _rows(), _rows(**bad)
    a = _shape(n_heads=8, n_kv_heads=8)
    assert _prompt(lib, a, (5, 1), [r, r, r, x]) == INVALID
    for at in (5, 6, 7):
        rows = [r] * 8
        rows[at] = x
        assert _grad(lib, a, (5, 1), rows) == INVALID, at
    c = _pages(n_seqs=100, table_stride=1)
    assert lib.opattr_attn_paged_window(c, 8, 5, 1, r, FAKE, 0.1, x, FAKE, None, FAKE, BIG,
                                        None) == INVALID
    c = _scaled(n_seqs=100, table_stride=1)
    assert lib.opattr_attn_paged_scaled(c, 8, 5, 1, r, FAKE, 0.1, x, FAKE, None, FAKE, BIG,
                                        None) == INVALID


def test_window_calls_past_their_places_or_one_launch_are_refused(lib):  # noqa: F811
    """Places and windows past them stay in 32 bits; a launch takes fewer than 2^32
    threads."""
    r = _rows()
    for a in (_shape(n_q=1 << 29), _shape(n_k=1 << 29),
              _shape(n_heads=64, n_kv_heads=64, n_seqs=1 << 19)):
        assert _prompt(lib, a, (5, 1), [r] * 4) == INVALID
        assert lib.opattr_attn_prompt_window_grad_workspace_bytes(a, 5, 1) == 0
        assert _grad(lib, a, (5, 1), [r] * 8) == INVALID
    assert lib.opattr_attn_prompt_window_grad_workspace_bytes(
        _shape(n_q=(1 << 29) - 1, n_k=(1 << 29) - 1, n_heads=2), 2 ** 31 - 1, 2 ** 31 - 1) > 0


def test_window_workspaces(lib):  # noqa: F811
    r, a = _rows(), _shape(n_q=5000, n_k=5000)
    for w in ((5, 0), (5, 1), (2 ** 31 - 1, 2 ** 31 - 1)):
        need = lib.opattr_attn_prompt_window_grad_workspace_bytes(a, *w)
        assert need >= 5000 * 8 * 8
        for ws, n in ((None, need), (FAKE, need - 1), (FAKE + 16, need)):
            assert _grad(lib, a, w, [r] * 8, ws=ws, n=n) == WORKSPACE
        assert _grad(lib, a, w, [r] * 8, lse=None) == INVALID
    # a window that no share is larger than needs no room for partial results; the cache
    # of 8 bits counts it by whole runs of 16 tokens
    for c, need, none, some in (
            (_pages(table_stride=500), lib.opattr_attn_paged_window_workspace_bytes, (200, 56),
             (200, 57)),
            (_scaled(table_stride=500), lib.opattr_attn_paged_scaled_workspace_bytes, (193, 33),
             (194, 33))):
        assert need(c, 8, *none) == 0 < need(c, 8, *some) <= need(c, 8, 2 ** 31 - 1, 5)
    for c, call, need in (
            (_pages(table_stride=500), lib.opattr_attn_paged_window,
             lib.opattr_attn_paged_window_workspace_bytes),
            (_scaled(table_stride=500), lib.opattr_attn_paged_scaled,
             lib.opattr_attn_paged_scaled_workspace_bytes)):
        n = need(c, 8, 1000, 0)
        for ws, have in ((None, n), (FAKE, n - 1), (FAKE + 16, n)):
            assert call(c, 8, 1000, 0, r, FAKE, 0.1, r, FAKE, None, ws, have, None) == WORKSPACE


@pytest.mark.parametrize("bad", BAD_PAGES, ids=str)
def test_paged_window_refuses_pages(lib, bad):  # noqa: F811
    r, c = _rows(), _pages(**bad)
    assert lib.opattr_attn_paged_window(c, 8, 5, 1, r, FAKE, 0.1, r, FAKE, None, FAKE, BIG,
                                        None) == INVALID
    assert lib.opattr_attn_paged_window_workspace_bytes(c, 8, 5, 1) == 0


def _scaled(**kw):
    a = dict(k=FAKE, v=FAKE, page_stride=2048, token_stride=128, head_stride=64, k_scale=FAKE + 1,
             v_scale=FAKE + 3, scale_page_stride=8, scale_block_stride=2, scale_head_stride=1,
             n_pages=10, page_size=16, block_size=4, table=FAKE, n_seqs=3, table_stride=5,
             n_kv_heads=2, head_dim=64, dtype=0)
    a.update(kw)
    return attn.opattr_kv_scaled(**a)


BAD_SCALED = [dict(k=None), dict(v=None), dict(k=FAKE + 8), dict(v=FAKE + 4), dict(k_scale=None),
              dict(v_scale=None), dict(page_stride=2056), dict(page_stride=-16),
              dict(token_stride=-16), dict(token_stride=72), dict(head_stride=8),
              dict(scale_page_stride=-1), dict(scale_block_stride=-2), dict(scale_head_stride=-1),
              dict(scale_page_stride=1 << 41), dict(page_stride=1 << 41), dict(n_pages=-1),
              dict(page_size=0), dict(page_size=24), dict(page_size=2048), dict(block_size=0),
              dict(block_size=3), dict(block_size=32), dict(block_size=-4), dict(table=None),
              dict(n_seqs=-1), dict(n_seqs=1 << 20), dict(table_stride=-1),
              dict(table_stride=1 << 28), dict(n_kv_heads=0), dict(head_dim=8), dict(head_dim=72),
              dict(head_dim=144), dict(dtype=-1), dict(dtype=2)]


@pytest.mark.parametrize("bad", BAD_SCALED, ids=str)
def test_scaled_refuses_caches(lib, bad):  # noqa: F811
    r, c = _rows(), _scaled(**bad)
    assert lib.opattr_attn_paged_scaled(c, 8, 5, 1, r, FAKE, 0.1, r, FAKE, None, FAKE, BIG,
                                        None) == INVALID
    assert lib.opattr_kv_append_scaled(c, 3, FAKE, r, r, FAKE, None, None, None) == INVALID
    assert lib.opattr_attn_paged_scaled_workspace_bytes(c, 8, 5, 1) == 0


def test_scaled_refuses(lib):  # noqa: F811
    r, c = _rows(), _scaled(table_stride=500)
    call = lib.opattr_attn_paged_scaled
    for heads in (0, 3, 2 * 17):
        assert call(c, heads, 5, 1, r, FAKE, 0.1, r, FAKE, None, FAKE, BIG, None) == INVALID
    assert call(c, 8, 5, 1, r, None, 0.1, r, FAKE, None, FAKE, BIG, None) == INVALID
    assert call(c, 8, 5, 1, r, FAKE, float("nan"), r, FAKE, None, FAKE, BIG, None) == INVALID
    assert call(c, 8, 5, 1, _rows(hs=3), FAKE, 0.1, r, FAKE, None, FAKE, BIG, None) == INVALID
    assert call(c, 8, 5, 1, r, FAKE, 0.1, None, FAKE, None, FAKE, BIG, None) == INVALID
    assert call(_scaled(n_seqs=1 << 19), 32, 5, 1, r, FAKE, 0.1, r, FAKE, None, FAKE, BIG,
                None) == INVALID
    assert call(None, 8, 5, 1, r, FAKE, 0.1, r, FAKE, None, FAKE, BIG, None) == INVALID


def test_append_scaled_refuses(lib):  # noqa: F811
    r, c = _rows(), _scaled()
    call = lib.opattr_kv_append_scaled
    assert call(c, -1, FAKE, r, r, FAKE, None, None, None) == INVALID
    assert call(c, 3, None, r, r, FAKE, None, None, None) == INVALID
    assert call(c, 3, FAKE, r, r, None, None, None, None) == INVALID
    assert call(c, 3, FAKE, _rows(p=None), r, FAKE, None, None, None) == INVALID
    assert call(c, 3, FAKE, r, None, FAKE, None, None, None) == INVALID
    assert call(c, 3, FAKE, r, r, FAKE, FAKE, None, None) == INVALID  # lens_out is lens
    assert call(c, 1 << 27, FAKE, r, r, FAKE, None, None, None) == INVALID
    assert call(None, 3, FAKE, r, r, FAKE, None, None, None) == INVALID
    # more waves than one launch takes: 2^25 tokens in blocks of one, by two heads
    assert call(_scaled(block_size=1, scale_page_stride=32), 1 << 25, FAKE, r, r, FAKE, None, None,
                None) == INVALID


def test_scaled_caches_that_overlap_themselves_are_refused(lib):  # noqa: F811
    r = _rows()
    for bad in (dict(page_stride=0), dict(token_stride=0), dict(head_stride=0),
                dict(token_stride=64), dict(page_stride=1920), dict(head_stride=48),
                dict(scale_page_stride=0), dict(scale_block_stride=0), dict(scale_head_stride=0),
                dict(scale_block_stride=1), dict(scale_page_stride=7)):
        assert lib.opattr_kv_append_scaled(_scaled(**bad), 3, FAKE, r, r, FAKE, None, None,
                                           None) == INVALID, bad


def test_scaled_struct_matches_header(tmp_path):
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "opattr_attn.h"',
             "int main(void) {", '  printf("size %zu\\n", sizeof(opattr_kv_scaled));']
    fields = attn.opattr_kv_scaled._fields_
    lines += [f'  printf("{f} %zu\\n", offsetof(opattr_kv_scaled, {f}));' for f, _ in fields]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines + ["  return 0;", "}"]) + "\n")
    subprocess.run(["gcc", "-std=c11", "-I", os.path.dirname(HEADER), "-o", str(exe), str(src)],
                   check=True)
    got = dict(line.split() for line in subprocess.run([str(exe)], check=True, capture_output=True,
                                                       text=True).stdout.splitlines())
    assert int(got["size"]) == C.sizeof(attn.opattr_kv_scaled)
    for f, _ in fields:
        assert int(got[f]) == getattr(attn.opattr_kv_scaled, f).offset, f


# --------------------------------------------------------------------------- #
# the oracle                                                                  #
# --------------------------------------------------------------------------- #


@pytest.mark.parametrize("n,m,window,sinks", [(6, 6, 2, 0), (6, 6, 2, 1), (4, 9, 3, 2),
                                              (9, 4, 2, 1), (5, 5, 100, 0), (7, 7, 1, 3)])
def test_window_oracle_against_loops_and_differences(n, m, window, sinks):
    rng = np.random.default_rng(n * 10 + m)
    d, scale = 8, 0.3
    q, k, v = rng.normal(size=(n, d)), rng.normal(size=(m, d)), rng.normal(size=(m, d))
    dout = rng.normal(size=(n, d))

    def loss(q, k, v):
        s = 0.0
        for i in range(n):
            p = i + m - n
            js = [j for j in range(p + 1) if p - j < window or j < sinks]
            w = [np.exp(scale * q[i] @ k[j]) for j in js]
            for j, x in zip(js, w):
                s += x / sum(w) * (v[j] @ dout[i])
        return s

    got = W.head(q, k, v, scale, W.visible(n, m, window, sinks), "bfloat16", dout)
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


def test_window_oracle_bounds_fail_a_wrong_result():
    """The bounds are narrow enough to catch a window or sinks off by one."""
    rng = np.random.default_rng(3)
    n, d = 60, 64
    q, k, v, dout = (rng.normal(size=(n, d)) for _ in range(4))

    def at(window, sinks):
        return W.head(q, k, v, 0.125, W.visible(n, n, window, sinks), "bfloat16", dout)

    good = at(20, 3)
    for bad in (at(21, 3), at(19, 3), at(20, 2), at(20, 4)):
        for name in ("out", "dq", "dk", "dv"):
            value, bound = good[name]
            assert (np.abs(bad[name][0] - value) > bound).any(), name


def test_codes_against_torch():
    """The codes' values and the rounding to them are torch's float8_e4m3fn."""
    import torch

    e4m3 = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(e4m3, W.CODES)
    rng = np.random.default_rng(4)
    x = np.concatenate([rng.normal(size=4000) * 2.0 ** rng.integers(-14, 8, 4000), e4m3,
                        (e4m3[1:127] + e4m3[:126]) / 2, [2.0 ** -10, 3 * 2.0 ** -10, 448, -448]])
    x = np.clip(np.nan_to_num(x), -448, 448).astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(W.code_of(x), want)
    assert (W.code_of([np.nan, np.inf, -np.inf]) & 127 == 127).all()
    s = np.array([0, 1, 127, 247, 254, 255], np.uint8)
    got = W.values_of(np.full((6, 1), 0x38, np.uint8), s)[:, 0]
    want = torch.from_numpy(s).view(torch.float8_e8m0fnu).double().numpy()
    np.testing.assert_array_equal(got, want)


def test_scaled_oracle_against_values():
    """Appends keep every value within half a step of its block's scale, and the
    attention over them is attention over those values."""
    rng = np.random.default_rng(5)
    pages, page, heads, d = 4, 8, 2, 16
    codes = np.full((pages, page, heads, d), 0x7f, np.uint8)
    scales = np.full((pages, 2, heads), 255, np.uint8)
    table = np.array([[2, 0, 3]])
    x = rng.normal(size=(21, heads, d)) * 2.0 ** rng.integers(-6, 6, (21, heads, 1))
    at = 0
    for n in (3, 1, 9, 7, 1):
        codes, scales, bad = W.append_scaled(codes, scales, x[at:at + n], [0, n], table, [at])
        at += n
        assert bad == 0
    t = np.arange(21)
    for h in range(heads):
        c, s = codes[table[0, t // page], t % page, h], scales[table[0, t // page], t % page // 4, h]
        v = W.values_of(c, s)
        step = 2.0 ** (s.astype(np.float64) - 127)
        # half of a mantissa step, or of the smallest one, and again where a block grew
        assert (np.abs(v - x[:, h]) <= 2 * np.maximum(np.abs(x[:, h]) / 16, 2.0 ** -10 *
                                                      step[:, None])).all()
        assert (np.abs(v).max(1) <= 448 * step).all()
        q = rng.normal(size=d)
        seen = W.visible(1, 21, 9, 2)
        (out, _), (lse, _) = W.head_scaled(q, c, s, c, s, 0.25, seen[0], "bfloat16")
        one = W.head(q[None], v, v, 0.25, seen, "bfloat16")
        np.testing.assert_allclose(out, one["out"][0][0], rtol=1e-12)
        np.testing.assert_allclose(lse, one["lse"][0][0], rtol=1e-12)
    # a block without tokens of the sequence takes nothing from what it held
    assert W.append_scaled(codes, np.full_like(scales, 254), x[:1], [0, 1], table, [8])[1][0, 0, 0] \
        == W.exponent_of(x[0, 0]) + 127
