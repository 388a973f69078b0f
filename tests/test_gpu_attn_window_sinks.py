"""The gradient of window attention where blocks share the sinks' key tiles of some of a
batch's sequences, against the 64-bit oracle."""
import numpy as np
import pytest

from test_gpu_attn import DEV, _ints, _torch
from test_gpu_attn_window import _case, _check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,dtype", [(64, "bfloat16"), (128, "float16"), (72, "bfloat16")])
@pytest.mark.parametrize("sinks", [1, 130, 400])
def test_sinks_of_long_and_short_sequences(sinks, d, dtype):
    """Long sequences whose tiles are shared beside those whose are not, and none."""
    _check(_case([900, 5, 1100, 0, 40, 700], [900, 30, 1300, 7, 0, 640], 8, 2, d, 60, sinks,
                 dtype))


@pytest.mark.parametrize("h,g", [(8, 1), (16, 4)])
@pytest.mark.parametrize("n", [65, 130])
def test_sinks_of_many_sequences(n, h, g):
    """The shared tiles' slots, counted through more sequences than a wave has lanes."""
    rng = np.random.default_rng(n)
    lens = [int(x) for x in rng.integers(0, 9, n)]
    for at in (0, 3, 62, 63, 64, n - 1):
        lens[at] = int(rng.integers(300, 700))
    _check(_case(lens, lens, h, g, 64, 40, 131, "bfloat16"))


def test_sinks_in_buffers_of_more_rows():
    """Rows beside the sequences leave room for slots that no tile takes; they stay as they
    were, and the workspace's old contents say nothing."""
    torch = _torch()
    from paper_2609_11938_amd import attn

    s = _case([500, 620], [500, 620], 8, 2, 64, 50, 140, "bfloat16")
    out, lse, want = _check(s)

    def wide(t):
        w = torch.full((3000,) + t.shape[1:], float("nan"), dtype=t.dtype, device=DEV)
        w[700:1820] = t
        return w

    args = [wide(s[n]) for n in "qkv"]
    l2 = torch.zeros(8, 3000, device=DEV)
    l2[:, 700:1820] = lse
    cu, first = _ints([700, 1200, 1820]), None
    for fill in (0.0, float("nan")):
        ws = attn.Workspace(DEV)
        new = [torch.full_like(t, 7.0) for t in args]
        call = dict(scale=s["scale"], dq=new[0], dk=new[1], dv=new[2], ws=ws)
        for _ in range(2):
            attn.opattr_attn_prompt_window_grad(wide(s["do"]), *args, wide(out), l2, cu, 50, 140,
                                                **call)
            torch.cuda.synchronize()
            got = [t.clone() for t in new]
            ws.buf.view(torch.float32).fill_(fill)
        for name, t in zip(("dq", "dk", "dv"), got):
            assert (t[:700] == 7).all() and (t[1820:] == 7).all()
            off = np.abs(t[700:1820].double().cpu().numpy() - want[name][0])
            assert (off <= want[name][1]).all(), name
        assert first is None or all(torch.equal(t, u) for t, u in zip(got, first))
        first = got
