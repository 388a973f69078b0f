"""Window attention on the GPU against the 64-bit oracle (tests/attn_window_oracle.py)
and its bounds: prompts, their gradient and the paged cache, at the windows, sinks,
sizes and layouts where they can go wrong."""
import math

import numpy as np
import pytest

import attn_oracle as O
import attn_window_oracle as W
from paper_2609_11938_amd import attn, opattr
from test_gpu_attn import (DATA, DEV, _cache, _cu, _dt, _host, _ints, _layout, _prompt, _rand,
                           _torch, _within)

pytestmark = pytest.mark.gpu


def _case(lens_q, lens_k, h, g, d, window, sinks, dtype, layout="plain", seed=0, **kw):
    s = _prompt(lens_q, lens_k, h, g, d, True, dtype, layout, seed=seed, **kw)
    print(f"  window={window} sinks={sinks}", flush=True)
    s.update(window=window, sinks=sinks, layout=layout)
    return s


def _check(s, grad=True):
    torch = _torch()
    args, layout = (s["q"], s["k"], s["v"]), s["layout"]
    win = (s["window"], s["sinks"])
    kw = dict(cu_k=s["cu_k"], scale=s["scale"])
    diag = attn.new_diag(DEV)
    out0 = _layout(torch.full(s["q"].shape, float("nan"), dtype=s["q"].dtype, device=DEV), layout)
    out, lse = attn.opattr_attn_prompt_window(*args, s["cu_q"], *win, out=out0, diag=diag, **kw)
    torch.cuda.synchronize()
    want = W.packed(s["qh"], s["kh"], s["vh"], s["hq"], s["hk"], s["scale"], *win, s["dtype"],
                    s["doh"], _host(out))
    _within(out, want["out"], "out")
    _within(lse, want["lse"], "lse")
    if grad:
        new = [_layout(torch.full(t.shape, float("nan"), dtype=t.dtype, device=DEV), layout)
               for t in args]
        got = attn.opattr_attn_prompt_window_grad(s["do"], *args, out, lse, s["cu_q"], *win,
                                                  dq=new[0], dk=new[1], dv=new[2], diag=diag, **kw)
        torch.cuda.synchronize()
        for name, t in zip(("dq", "dk", "dv"), got):
            _within(t, want[name], name)
        again = attn.opattr_attn_prompt_window_grad(s["do"], *args, out, lse, s["cu_q"], *win,
                                                    **kw)
        for name, t, u in zip(("dq", "dk", "dv"), got, again):
            assert torch.equal(t, u), f"{name}: runs differ"
    assert opattr.read_diag(diag)["status"] == 0
    return out, lse, want


SEQS = [([1], [1]), ([5], [5]), ([129], [129]), ([31, 0, 260, 2], [31, 0, 260, 2]),
        ([1, 1, 1], [300, 65, 1]), ([100, 40], [37, 0]), ([3, 170], [200, 450])]


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (33, 0), (64, 4), (100, 70),
                                          (1000, 3), (7, 1000)])
@pytest.mark.parametrize("lens", SEQS, ids=str)
def test_window_lengths(lens, window, sinks):
    _check(_case(*lens, 4, 2, 64, window, sinks, "bfloat16"))


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("h,g,d", [(1, 1, 8), (3, 1, 24), (6, 3, 72), (4, 4, 128), (8, 1, 128),
                                   (5, 5, 120)])
def test_window_heads(h, g, d, dtype):
    _check(_case([70, 331], [70, 331], h, g, d, 90, 5, dtype))


@pytest.mark.parametrize("sinks", [0, 1, 31, 32, 33, 63, 64, 65, 128, 130, 200])
@pytest.mark.parametrize("window", [31, 32, 64, 65, 127, 128, 129])
def test_window_edges(window, sinks):
    """Windows and sinks that end on, before and after a tile's last key, in queries
    and heads of both tile sizes."""
    _check(_case([420], [420], 2, 1, 128, window, sinks, "bfloat16"))
    _check(_case([200], [460], 2, 2, 40, window, sinks, "float16"))


@pytest.mark.parametrize("layout", ["heads", "packed"])
@pytest.mark.parametrize("d,dtype", [(64, "float16"), (128, "bfloat16"), (40, "bfloat16")])
def test_window_layouts(layout, d, dtype):
    _check(_case([90, 7, 230], [90, 7, 230], 4, 2, d, 50, 6, dtype, layout))


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window,sinks", [(257, 4), (800, 4), (900, 0)])
def test_window_long(d, dtype, window, sinks):
    """Two groups of waves share the keys where the window is long."""
    _check(_case([1500, 1115], [1500, 1377], 2, 1, d, window, sinks, dtype))


@pytest.mark.parametrize("n", [65, 130])
@pytest.mark.parametrize("dtype,d", [("bfloat16", 64), ("float16", 128)])
def test_window_many_sequences(n, dtype, d):
    rng = np.random.default_rng(n)
    lens = [int(x) for x in rng.integers(0, 9, n)]
    for at in (1, 63, 64, n - 1):
        lens[at] = int(rng.integers(150, 300))
    keys = [x + (b % 3) * 50 for b, x in enumerate(lens)]
    keys[5] = 0
    _check(_case(lens, keys, 4, 2, d, 40, 3, dtype))


@pytest.mark.parametrize("window,sinks,h,g", [(128, 4, 8, 1), (300, 0, 16, 1), (200, 130, 12, 2)])
def test_window_split_key_tiles(window, sinks, h, g):
    """Key tiles shared by blocks: the sinks' own tiles, which every query meets."""
    s = _case([1400, 300], [1400, 300], h, g, 64, window, sinks, "bfloat16")
    _check(s)


@pytest.mark.parametrize("lens", [[1300, 40], [1, 900, 1, 1]], ids=str)
@pytest.mark.parametrize("window,sinks", [(449, 0), (449, 3), (670, 3), (671, 3), (671, 200),
                                          (5000, 140)])
def test_window_near_the_mean_length(lens, window, sinks):
    """Windows on both sides of the sequences' mean length, where the gradient's key tiles
    begin to be split as the causal mask's are."""
    _check(_case(lens, lens, 8, 2, 64, window, sinks, "bfloat16"))


@pytest.mark.parametrize("n,window,sinks", [(64, 13, 0), (64, 13, 5), (300, 100, 0),
                                            (521, 773, 0), (521, 200, 130)])
@pytest.mark.parametrize("d,dtype", [(64, "bfloat16"), (128, "float16")])
def test_window_one_sequence_of_many_heads(n, window, sinks, d, dtype):
    """One key head, whose few key tiles are split into blocks of few steps."""
    _check(_case([n], [n], 8, 1, d, window, sinks, dtype))


def test_window_as_long_as_the_sequences_is_the_causal_mask():
    """By the bounds of attention without a window: which of two products joins a sum by
    a fused operation is the compiler's choice in each kernel, so bits may differ."""
    for lens, d, dtype in (([900], 64, "float16"), ([130, 61, 0, 300], 128, "bfloat16")):
        s = _case(lens, lens, 4, 2, d, 1 << 30, 0, dtype)
        args = (s["q"], s["k"], s["v"])
        for window, sinks in ((1 << 30, 0), (1 << 40, 1 << 40), (max(lens), 0)):
            out, lse = attn.opattr_attn_prompt_window(*args, s["cu_q"], window, sinks,
                                                      scale=s["scale"])
            want = O.packed(s["qh"], s["kh"], s["vh"], s["hq"], s["hk"], s["scale"], True, dtype,
                            s["doh"], _host(out))
            _within(out, want["out"], "out")
            _within(lse, want["lse"], "lse")
            got = attn.opattr_attn_prompt_window_grad(s["do"], *args, out, lse, s["cu_q"], window,
                                                      sinks, scale=s["scale"])
            for name, t in zip(("dq", "dk", "dv"), got):
                _within(t, want[name], name)
    rng = np.random.default_rng(1)
    lens = [700, 0, 31, 1200]
    cache, table, kv = _cache(rng, lens, 2, 64, 16, "bfloat16")
    q, qh = _rand(rng, (4, 4, 64), "bfloat16")
    for window, sinks in ((1 << 30, 0), (2000, 5), (1200, 0)):
        out, lse = attn.opattr_attn_paged_window(q, cache[0], cache[1], _ints(table), _ints(lens),
                                                 window, sinks)
        for b in range(4):
            for j in range(4):
                one = O.head(qh[b:b + 1, j], kv[b][0][:, j // 2], kv[b][1][:, j // 2], 0.125,
                             False, "bfloat16")
                _within(out[b:b + 1, j], one["out"], f"out[{b}, {j}]")
                _within(lse[j, b:b + 1], one["lse"], f"lse[{j}, {b}]")


def test_window_sharp_and_flat():
    _check(_case([300], [300], 2, 2, 64, 70, 4, "bfloat16", gain=30.0))
    _check(_case([300], [300], 2, 2, 64, 70, 4, "float16", scale=0.0))
    _check(_case([250], [250], 2, 1, 64, 33, 40, "float16", scale=-0.2))


def test_window_nothing():
    torch = _torch()
    z = torch.zeros(0, 2, 64, dtype=torch.bfloat16, device=DEV)
    out, lse = attn.opattr_attn_prompt_window(z, z, z, _ints([0]), 5)
    assert out.shape == (0, 2, 64) and lse.shape == (2, 0)
    got = attn.opattr_attn_prompt_window_grad(z, z, z, z, out, lse, _ints([0, 0]), 5, 1)
    assert all(t.numel() == 0 for t in got)
    k = torch.ones(10, 1, 64, dtype=torch.bfloat16, device=DEV)
    out, lse = attn.opattr_attn_prompt_window(z, k, k, _ints([0, 0]), 5, cu_k=_ints([0, 10]))
    _, dk, dv = attn.opattr_attn_prompt_window_grad(z, z, k, k, out, lse, _ints([0, 0]), 5,
                                                    cu_k=_ints([0, 10]))
    assert (dk == 0).all() and (dv == 0).all()


def test_window_empty_rows_are_zero():
    s = _case([50, 20], [30, 0], 2, 1, 64, 8, 2, "bfloat16")
    out, lse, _ = _check(s)
    assert (out[:20] == 0).all() and (out[50:] == 0).all()
    assert _torch().isneginf(lse[:, :20]).all() and _torch().isneginf(lse[:, 50:]).all()


@pytest.mark.parametrize("what", [float("nan"), float("inf"), 3e38])
@pytest.mark.parametrize("window,sinks,n", [(50, 4, 240), (800, 3, 1000)])
def test_window_hidden_values_do_not_matter(what, window, sinks, n):
    """Values that no finite sum survives, at a key that only some queries see: those
    before it, and those whose window has left it, have the same bits."""
    torch = _torch()
    s = _case([n], [n], 2, 1, 64, window, sinks, "bfloat16")
    out, lse, want = _check(s, grad=False)
    for row in (sinks, 70, 130, n - 1):
        k, v = s["k"].clone(), s["v"].clone()
        v[row] = k[row] = what
        got, gl = attn.opattr_attn_prompt_window(s["q"], k, v, s["cu_q"], window, sinks,
                                                 scale=s["scale"])
        free = np.r_[0:row, min(row + window, n):n]
        _within(got[free], tuple(t[free] for t in want["out"]), f"out beside {row}")
        assert torch.equal(gl[:, free], lse[:, free]), row
        if math.isnan(what):
            assert torch.isnan(got[row:row + window]).all()
    # a sink is seen by every query from it on
    k = s["k"].clone()
    k[0] = float("nan")
    got, _ = attn.opattr_attn_prompt_window(s["q"], k, s["v"], s["cu_q"], window, sinks)
    assert torch.isnan(got).all()


def test_window_rows_beside_sequences():
    """Neither read nor written."""
    torch = _torch()
    s = _case([140], [140], 2, 1, 64, 30, 3, "float16")
    out, lse, want = _check(s, grad=False)
    dq, _, _ = attn.opattr_attn_prompt_window_grad(s["do"], s["q"], s["k"], s["v"], out, lse,
                                                   s["cu_q"], 30, 3, scale=s["scale"])

    def wide(t, beside):
        w = torch.full((300,) + t.shape[1:], beside, dtype=t.dtype, device=DEV)
        w[100:240] = t
        return w

    cu, first = _ints([100, 240]), None
    for beside in (float("nan"), 3.0):
        args = [wide(s[n], beside) for n in "qkv"]
        o2, l2 = torch.full_like(args[0], 7.0), torch.full((2, 300), 7.0, device=DEV)
        attn.opattr_attn_prompt_window(*args, cu, 30, 3, scale=s["scale"], out=o2, lse=l2)
        assert torch.equal(o2[100:240], out) and torch.equal(l2[:, 100:240], lse)
        assert (o2[:100] == 7).all() and (o2[240:] == 7).all() and (l2[:, :100] == 7).all()
        new = [torch.full_like(t, 7.0) for t in args]
        attn.opattr_attn_prompt_window_grad(wide(s["do"], beside), *args, o2, l2, cu, 30, 3,
                                            scale=s["scale"], dq=new[0], dk=new[1], dv=new[2])
        # a query's sum has one order; a sink's is split by the rows that the buffers have,
        # 140 or 300, so its bits are those of buffers as large, its value the formula's
        assert torch.equal(new[0][100:240], dq)
        for name, t in zip(("dq", "dk", "dv"), new):
            assert (t[:100] == 7).all() and (t[240:] == 7).all()
            _within(t[100:240], want[name], name)
        assert first is None or all(torch.equal(t, u) for t, u in zip(new, first))
        first = new


def test_window_grad_against_differences():
    """The gradient times a direction against differences of the 64-bit loss."""
    win = (20, 3)
    s = _case([37, 66], [37, 90], 4, 2, 64, *win, "bfloat16")
    out, lse = attn.opattr_attn_prompt_window(s["q"], s["k"], s["v"], s["cu_q"], *win,
                                              cu_k=s["cu_k"], scale=s["scale"])
    got = attn.opattr_attn_prompt_window_grad(s["do"], s["q"], s["k"], s["v"], out, lse, s["cu_q"],
                                              *win, cu_k=s["cu_k"], scale=s["scale"])
    host = [s["qh"], s["kh"], s["vh"]]

    def loss(q, k, v):
        o = W.packed(q, k, v, s["hq"], s["hk"], s["scale"], *win, "bfloat16")["out"][0]
        return (o * s["doh"]).sum()

    want = W.packed(*host, s["hq"], s["hk"], s["scale"], *win, "bfloat16", s["doh"], _host(out))
    rng = np.random.default_rng(1)
    for at, name in enumerate(("dq", "dk", "dv")):
        way = rng.normal(size=host[at].shape)
        up, down = list(host), list(host)
        h = 1e-5
        up[at], down[at] = host[at] + h * way, host[at] - h * way
        diff = (loss(*up) - loss(*down)) / (2 * h)
        bound = (want[name][1] * np.abs(way)).sum() + 1e-5 * abs(diff) + 1e-7
        assert abs((_host(got[at]) * way).sum() - diff) <= bound, name


@pytest.mark.parametrize("dtype,gain", [("float16", 2e-4), ("bfloat16", 1e-12), ("float16", 300.0)])
def test_window_grad_small_and_large(dtype, gain):
    s = _case([190], [190], 2, 1, 64, 40, 4, dtype)
    s["do"] = (s["do"].float() * gain).to(s["do"].dtype)
    s["doh"] = _host(s["do"])
    _check(s)


@pytest.mark.parametrize("d", [64, 128])
def test_window_grad_hidden_finite_values(d):
    """A finite value whose product with dout no float32 holds, at a key that queries
    with a gradient no longer see."""
    torch = _torch()
    s = _case([300], [300], 2, 1, d, 60, 4, "bfloat16")
    s["v"] = s["v"].clone()
    s["v"][100] = 1e36
    s["do"] = s["do"] * 1e3
    s["do"][100:160] = 0
    s["vh"], s["doh"] = _host(s["v"]), _host(s["do"])
    assert not torch.isfinite(s["do"][200:, 0].float() @ s["v"][100, 0].float()).any()
    _check(s)


def test_window_bad_offsets_are_flagged():
    torch = _torch()
    s = _case([60, 40], [60, 40], 2, 1, 64, 20, 2, "bfloat16")
    for cu in ([0, 60, 150], [-5, 60, 100], [0, 70, 60]):
        diag = attn.new_diag(DEV)
        out, lse = attn.opattr_attn_prompt_window(s["q"], s["k"], s["v"], _ints(cu), 20, 2,
                                                  diag=diag)
        torch.cuda.synchronize()
        assert opattr.read_diag(diag)["status"] == DATA, cu


def test_window_graph_replays():
    """Captured with buffers of the caller's, replayed with new inputs between eager
    work: every replay as the eager call."""
    torch = _torch()
    s = _case([80, 330], [80, 330], 8, 1, 64, 50, 4, "float16")
    q, k, v, do, cu = s["q"], s["k"], s["v"], s["do"], s["cu_q"]
    ws = attn.Workspace(DEV)
    out, lse = attn.opattr_attn_prompt_window(q, k, v, cu, 50, 4)
    g = attn.opattr_attn_prompt_window_grad(do, q, k, v, out, lse, cu, 50, 4, ws=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        attn.opattr_attn_prompt_window(q, k, v, cu, 50, 4, out=out, lse=lse)
        attn.opattr_attn_prompt_window_grad(do, q, k, v, out, lse, cu, 50, 4, dq=g[0], dk=g[1],
                                            dv=g[2], ws=ws)
    for turn in range(3):
        q.mul_(0.7)
        do.mul_(0.5)
        want, wl = attn.opattr_attn_prompt_window(q, k, v, cu, 50, 4)
        wg = attn.opattr_attn_prompt_window_grad(do, q, k, v, want, wl, cu, 50, 4)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, wl), turn
        assert all(torch.equal(a, b) for a, b in zip(g, wg)), turn


def test_window_other_stream():
    torch = _torch()
    s = _case([300, 200], [300, 200], 4, 2, 64, 60, 4, "bfloat16")
    args, cu = (s["q"], s["k"], s["v"]), s["cu_q"]
    want, wl = attn.opattr_attn_prompt_window(*args, cu, 60, 4)
    grads = attn.opattr_attn_prompt_window_grad(s["do"], *args, want, wl, cu, 60, 4)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out, lse = attn.opattr_attn_prompt_window(*args, cu, 60, 4, stream=side)
    got = attn.opattr_attn_prompt_window_grad(s["do"], *args, out, lse, cu, 60, 4, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(lse, wl)
    assert all(torch.equal(t, u) for t, u in zip(got, grads))


def test_paged_window_other_stream():
    torch = _torch()
    rng = np.random.default_rng(3)
    lens = [900, 70]
    cache, table, _ = _cache(rng, lens, 2, 64, 16, "bfloat16")
    q, _ = _rand(rng, (2, 4, 64), "bfloat16")
    args = (q, cache[0], cache[1], _ints(table), _ints(lens), 400, 5)
    want, wl = attn.opattr_attn_paged_window(*args)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out, lse = attn.opattr_attn_paged_window(*args, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(lse, wl)


def test_window_binding_refuses():
    torch = _torch()
    s = _case([20], [20], 2, 1, 64, 5, 1, "bfloat16")
    q, k, v, cu = s["q"], s["k"], s["v"], s["cu_q"]
    out, lse = attn.opattr_attn_prompt_window(q, k, v, cu, 5, 1)
    pages = torch.zeros(2, 3, 16, 1, 64, dtype=torch.bfloat16, device=DEV)
    table, lens = _ints([[0, 1]]), _ints([20])
    for window, sinks in ((0, 0), (-1, 0), (5, -1), (1.5, 0), (5, None)):
        for call in (lambda: attn.opattr_attn_prompt_window(q, k, v, cu, window, sinks),
                     lambda: attn.opattr_attn_prompt_window_grad(s["do"], q, k, v, out, lse, cu,
                                                                 window, sinks),
                     lambda: attn.opattr_attn_paged_window(q[:1], pages[0], pages[1], table, lens,
                                                           window, sinks)):
            with pytest.raises((TypeError, ValueError, RuntimeError)):
                call()
    bad = [lambda: attn.opattr_attn_prompt_window(q.float(), k.float(), v.float(), cu, 5),
           lambda: attn.opattr_attn_prompt_window(q, k, v[:10], cu, 5),
           lambda: attn.opattr_attn_prompt_window(q, k, v, cu, 5, cu_k=_ints([0, 10, 20])),
           lambda: attn.opattr_attn_paged_window(q[:1], pages[0], pages[1].half(), table, lens, 5),
           lambda: attn.opattr_attn_paged_window(q[:2], pages[0], pages[1], table, lens, 5)]
    for f in bad:
        with pytest.raises((TypeError, ValueError, RuntimeError)):
            f()
    for t in (q, k, v):
        t.requires_grad_()
        with pytest.raises(RuntimeError, match="grad"):
            attn.opattr_attn_prompt_window(q, k, v, cu, 5, 1)
        t.requires_grad_(False)
    torch.cuda.synchronize()


# --------------------------------------------------------------------------- #
# paged cache                                                                 #
# --------------------------------------------------------------------------- #


def _check_paged(lens, h, g, d, page, window, sinks, dtype, order="nhd", ws=None):
    torch = _torch()
    print(f"case paged window={window} sinks={sinks} lens={lens} heads={h}/{g} d={d} page={page} "
          f"{dtype} {order}", flush=True)
    rng = np.random.default_rng([h, g, d, page, len(lens), window])
    cache, table, kv = _cache(rng, lens, g, d, page, dtype, order=order)
    # entries of pages that the window has left behind say nothing, their values neither
    for b, n in enumerate(lens):
        for x in range(-(-n // page)):
            if x * page >= sinks and (x + 1) * page <= n - window:
                cache[:, table[b, x]] = float("nan")
                table[b, x] = (-1, 1 << 30, table[b, x])[x % 3]
    q, qh = _rand(rng, (len(lens), h, d), dtype, 2.0)
    scale = 1 / math.sqrt(d)
    diag = attn.new_diag(DEV)
    args = (q, cache[0], cache[1], _ints(table), _ints(lens), window, sinks)
    out, lse = attn.opattr_attn_paged_window(*args, diag=diag, ws=ws)
    torch.cuda.synchronize()
    for b, n in enumerate(lens):
        seen = W.visible(1, n, window, sinks)
        for j in range(h):
            one = W.head(qh[b:b + 1, j], kv[b][0][:, j * g // h], kv[b][1][:, j * g // h], scale,
                         seen, dtype)
            _within(out[b:b + 1, j], one["out"], f"out[{b}, {j}]")
            _within(lse[j, b:b + 1], one["lse"], f"lse[{j}, {b}]")
    assert opattr.read_diag(diag)["status"] == 0
    again, _ = attn.opattr_attn_paged_window(*args, ws=ws)
    assert torch.equal(out, again), "runs differ"


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("h,g,d,page", [(2, 2, 64, 16), (8, 2, 128, 16), (16, 1, 128, 32),
                                        (3, 1, 72, 1), (4, 4, 8, 64), (2, 1, 40, 1024)])
def test_paged_window_heads(h, g, d, page, dtype):
    _check_paged([1, 37, 0, 230], h, g, d, page, 50, 5, dtype)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (31, 1), (32, 0), (100, 4), (256, 0),
                                          (252, 4), (253, 4), (600, 300), (5, 1000)])
@pytest.mark.parametrize("lens", [[0], [1], [33], [257], [5000, 3, 0, 700], [1, 90] * 40],
                         ids=lambda v: str(v)[:30])
def test_paged_window_lengths(lens, window, sinks):
    _check_paged(lens, 4, 1, 64, 16, window, sinks, "bfloat16")


def test_paged_window_long_split():
    ws = attn.Workspace(DEV)
    _check_paged([40000], 4, 2, 64, 16, 20000, 100, "float16", ws=ws)
    _check_paged([20011, 1, 0, 300], 8, 2, 128, 64, 5000, 4, "bfloat16", ws=ws)
    _check_paged([100, 345], 4, 2, 64, 16, 77, 18, "bfloat16", order="hnd")


def test_paged_window_bad_table_and_lens():
    """Entries out of range among the pages that are seen are masked, lengths past the
    table cut; both flagged."""
    torch = _torch()
    rng = np.random.default_rng(5)
    lens, page, window, sinks = [90, 70], 16, 40, 20
    cache, table, kv = _cache(rng, lens, 2, 64, page, "bfloat16", width=7)
    q, qh = _rand(rng, (2, 4, 64), "bfloat16")
    for where, value, hit in (((0, 1), 10_000, 4), ((1, 3), -3, 16), ((0, 2), -1, 0)):
        bad = table.copy()
        bad[where] = value
        diag = attn.new_diag(DEV)
        out, lse = attn.opattr_attn_paged_window(q, cache[0], cache[1], _ints(bad), _ints(lens),
                                                 window, sinks, diag=diag)
        torch.cuda.synchronize()
        got = opattr.read_diag(diag)
        assert got["status"] == (DATA if hit else 0) and got["bad_records"] == hit
        b, x = where
        seen = W.visible(1, lens[b], window, sinks)
        seen[0, x * page:(x + 1) * page] = False
        one = W.head(qh[b:b + 1, 0], kv[b][0][:, 0], kv[b][1][:, 0], 0.125, seen, "bfloat16")
        _within(out[b:b + 1, 0], one["out"], "out")
        _within(lse[0, b:b + 1], one["lse"], "lse")
    cache.nan_to_num_(0.5)
    full = _ints(rng.permutation(cache.shape[1])[:12].reshape(2, 6))
    want, _ = attn.opattr_attn_paged_window(q, cache[0], cache[1], full, _ints([96, 0]), 40, 20)
    diag = attn.new_diag(DEV)
    got, _ = attn.opattr_attn_paged_window(q, cache[0], cache[1], full, _ints([9999, -7]), 40, 20,
                                           diag=diag)
    assert torch.equal(got, want) and opattr.read_diag(diag)["status"] == DATA


def test_window_steps_continue_a_prompt():
    """A prompt through the window, then its last tokens again one by one from the cache:
    the same outputs within both sides' bounds."""
    torch = _torch()
    n, page, window, sinks = 200, 16, 50, 4
    s = _case([n], [n], 4, 2, 64, window, sinks, "bfloat16")
    out, lse, want = _check(s, grad=False)
    cache = torch.full((2, 15, page, 2, 64), float("nan"), dtype=torch.bfloat16, device=DEV)
    table = _ints(np.random.default_rng(2).permutation(15)[None, :13])
    lens = _ints([0])
    for lo, hi in ((0, 150), *((t, t + 1) for t in range(150, n))):
        lens = attn.opattr_kv_append(s["k"][lo:hi], s["v"][lo:hi], _ints([0, hi - lo]), cache[0],
                                     cache[1], table, lens)
        if hi > 150:
            got, gl = attn.opattr_attn_paged_window(s["q"][lo:hi], cache[0], cache[1], table, lens,
                                                    window, sinks)
            _within(got, tuple(t[lo:hi] for t in want["out"]), f"out at {lo}")
            _within(gl, tuple(t[:, lo:hi] for t in want["lse"]), f"lse at {lo}")
