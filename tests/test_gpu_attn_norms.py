"""The gradient in float16 of batches of uneven lengths: the power of two that its products
are scaled by goes by the largest rows of each sequence and head, wherever they stand."""
import numpy as np
import pytest

import attn_oracle as O
import attn_window_oracle as W
from paper_2609_11938_amd import attn
from test_gpu_attn import _host, _prompt, _torch, _within

pytestmark = pytest.mark.gpu


def _steps_of_the_group(s, do, window):
    """What the oracle's bound of dk, made head by head, leaves out. dk takes the products
    of all query heads of a key head by one power of two, 2^e, with the group's largest
    |dout| |v| = M in [2^(13 - e), 2^(14 - e)): below 2^-14 a scaled ds is off by half of
    float16's smallest step, 2^-25, which is 2^(-25 - e) <= 2^-38 M of ds. The oracle has 2^-36
    with each head's own largest, so this has it with the group's."""
    q, v, cu, scale = s["qh"], _host(s["v"]), s["hq"], s["scale"]
    more = np.zeros(s["kh"].shape)
    group = q.shape[1] // v.shape[1]
    for b in range(len(cu) - 1):
        t = slice(cu[b], cu[b + 1])
        n = cu[b + 1] - cu[b]
        seen = W.visible(n, n, window or 1 << 30, 4)
        for g in range(v.shape[1]):
            h = slice(g * group, (g + 1) * group)
            most = np.linalg.norm(do[t, h], axis=2).max(initial=0.0) * \
                np.linalg.norm(v[t, g], axis=1).max(initial=0.0)
            more[t, g] = 2.0 ** -36 * scale * most * (seen.T @ np.abs(q[t, h]).sum(1))
    return more


@pytest.mark.parametrize("window", [None, 90])
@pytest.mark.parametrize("h,g,d", [(4, 2, 64), (3, 3, 128), (16, 1, 40)])
@pytest.mark.parametrize("at", [0, 127, 128, 640, 699])
def test_one_large_row(at, h, g, d, window):
    """Rows of dout and v far larger than the others, in one sequence and head: its own
    sums do not overflow, and the other sequences' small ones keep their bits."""
    torch = _torch()
    lens = [3, 700, 0, 128, 129, 1]
    s = _prompt(lens, lens, h, g, d, True, "float16")
    print(f"  at={at} window={window}", flush=True)
    s["do"] = (s["do"].float() * 2e-3).half()
    s["v"] = (s["v"].float() * 0.05).half()
    s["do"][3 + at, h - 1] *= 1e4
    s["v"][3 + 699 - at, g - 1] *= 100
    assert torch.isfinite(s["do"]).all() and torch.isfinite(s["v"]).all()
    host = [_host(s[n]) for n in ("q", "k", "v")]
    args, do = (s["q"], s["k"], s["v"]), _host(s["do"])
    for _ in range(2):  # the second in memory that the first one left
        if window:
            out, lse = attn.opattr_attn_prompt_window(*args, s["cu_q"], window, 4,
                                                      scale=s["scale"])
            got = attn.opattr_attn_prompt_window_grad(s["do"], *args, out, lse, s["cu_q"], window,
                                                      4, scale=s["scale"])
            want = W.packed(*host, s["hq"], s["hk"], s["scale"], window, 4, "float16", do,
                            _host(out))
        else:
            out, lse = attn.opattr_attn_prompt(*args, s["cu_q"], scale=s["scale"])
            got = attn.opattr_attn_prompt_grad(s["do"], *args, out, lse, s["cu_q"],
                                               scale=s["scale"])
            want = O.packed(*host, s["hq"], s["hk"], s["scale"], True, "float16", do, _host(out))
        want["dk"] = want["dk"][0], want["dk"][1] + _steps_of_the_group(s, do, window)
        for name, t in zip(("dq", "dk", "dv"), got):
            _within(t, want[name], name)


def test_long_sequences_of_many_pieces():
    """More pieces of a sequence than a wave has lanes; the largest row in the last."""
    torch = _torch()
    lens, h, g, d = [9000, 40], 2, 1, 64
    print("case", lens, flush=True)
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(4)
    n = sum(lens)
    q, k, v, do = (torch.randn(n, x, d, generator=gen, device="cuda:0").half()
                   for x in (h, g, g, h))
    do *= 1e-3
    do[8990, 1] *= 3e4
    v[8985] *= 30
    cu = torch.tensor([0, 9000, n], dtype=torch.int32, device="cuda:0")
    out, lse = attn.opattr_attn_prompt_window(q, k, v, cu, 30, scale=0.125)
    got = attn.opattr_attn_prompt_window_grad(do, q, k, v, out, lse, cu, 30, scale=0.125)
    # the last 60 queries' share, whose keys the sequence's last 89 are
    part = slice(8911, 9000)
    want = W.packed(*(_host(t[part]) for t in (q, k, v)), [0, 89], [0, 89], 0.125, 30, 0,
                    "float16", _host(do[part]), _host(out[part]))
    for name, t in zip(("dq", "dk", "dv"), got):
        value, bound = (x[29:] for x in want[name])
        _within(t[8940:9000], (value, bound), name)
    assert all(torch.isfinite(t).all() for t in got)
    small = W.packed(*(_host(t[9000:]) for t in (q, k, v)), [0, 40], [0, 40], 0.125, 30, 0,
                     "float16", _host(do[9000:]), _host(out[9000:]))
    for name, t in zip(("dq", "dk", "dv"), got):
        _within(t[9000:], small[name], name)
    assert np.abs(small["dq"][0]).max() > 0
