"""The attention workload through a window and with a cache of 8 bits: what it generates
and trains has the outputs of the definition, across a fork and a compaction, and its
launches carry the operators' names and bytes."""
import numpy as np
import pytest

import attn_window_oracle as W
from test_gpu_workload import _host

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("window,sinks", [(20, 3), (1, 0), (500, 2)])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_generated_tokens_through_a_window_match_whole_sequences(dtype, window, sinks):
    import torch

    from paper_2609_11938_amd import workload

    print(f"case serve {dtype} window={window} sinks={sinks}", flush=True)
    rec = workload.Recorder()
    alive = workload.serve(rec, lens=(50, 9, 33), steps=5, layers=2, heads=4, kv_heads=2,
                           head_dim=64, page_size=8, dtype=getattr(torch, dtype), window=window,
                           sinks=sinks)
    assert [seq[0][0].shape[0] for seq in alive] == [60, 60, 43]
    for seq in alive:
        for q, k, v, out in seq:
            q, k, v, out = (_host(t) for t in (q, k, v, out))
            seen = W.visible(len(q), len(q), window, sinks)
            for h in range(4):
                want, bound = W.head(q[:, h], k[:, h // 2], v[:, h // 2], 0.125, seen,
                                     dtype)["out"]
                assert (np.abs(out[:, h] - want) <= bound).all()
    assert {"attn_prompt_window", "attn_paged_window"} <= set(rec.names)
    assert "attn_paged" not in rec.names


@pytest.mark.parametrize("window,sinks", [(None, 0), (20, 3)])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_generation_from_a_cache_of_8_bits(dtype, window, sinks, monkeypatch):
    """The last step's outputs are those of the codes that the cache ends with, whose
    values are the rows that were appended, within their rounding."""
    import torch

    from paper_2609_11938_amd import workload

    print(f"case serve {dtype} scaled window={window} sinks={sinks}", flush=True)
    made = []

    class Kept(workload.Cache):
        def __init__(self, *args, **kw):
            super().__init__(*args, **kw)
            made.append(self)

    monkeypatch.setattr(workload, "Cache", Kept)
    rec = workload.Recorder()
    alive = workload.serve(rec, lens=(50, 9, 33), steps=5, layers=2, heads=4, kv_heads=2,
                           head_dim=64, page_size=8, dtype=getattr(torch, dtype), window=window,
                           sinks=sinks, scaled=True)
    cache, = made
    assert cache.lens.tolist() == [60, 60, 43]
    table, codes, scales = (t.cpu().numpy() for t in (cache.table, cache.data, cache.scales))
    for b, seq in enumerate(alive):
        n = seq[0][0].shape[0]
        t = np.arange(n)
        page, slot = table[b, t // 8], t % 8
        for layer, (q, k, v, out) in enumerate(seq):
            q, k, v, out = (_host(x) for x in (q, k, v, out))
            seen = W.visible(1, n, window or n, sinks)[0]
            for g in range(2):
                kc, vc = ((codes[layer, i][page, slot, g], scales[layer, i][page, 0, g])
                          for i in range(2))
                for x, (c, s) in ((k, kc), (v, vc)):
                    # half a step of 2^-3 of the value, or of the block's smallest; each
                    # growth, which doubles that at least, rounds once more
                    step = 2.0 ** (s.astype(np.float64) - 127)[:, None]
                    off = np.abs(W.values_of(c, s) - x[:, g])
                    assert (off <= np.abs(x[:, g]) / 16 + 2.0 ** -9 * step).all()
                for h in (2 * g, 2 * g + 1):
                    (want, bound), _ = W.head_scaled(q[-1, h], *kc, *vc, 0.125, seen, dtype)
                    assert (np.abs(out[-1, h] - want) <= bound).all()
    assert {"kv_append_scaled", "attn_paged_scaled", "pages_fork", "pages_compact"} <= \
        set(rec.names)
    tr = rec.trace()
    first = rec.names.index("kv_append_scaled")
    at = int(np.flatnonzero(tr["name_id"] == first)[0])
    rows = 2 * 92 * 2 * 64  # the prompts' keys and values
    assert tr["counters"][at, workload.READ] == 2 * rows
    assert tr["counters"][at, workload.WRITTEN] == rows


def test_training_through_a_window():
    import torch

    from paper_2609_11938_amd import workload

    rec = workload.Recorder()
    lens, window, sinks = (130, 77), 30, 2
    out, dq, dk, dv = workload.train(rec, lens=lens, window=window, sinks=sinks)
    assert rec.names == ["attn_prompt_window", "attn_prompt_window_grad"]
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(0)
    q, k, v = workload._rows(sum(lens), 8, 4, 64, gen, torch.bfloat16)
    do = torch.randn(q.shape, generator=gen, device="cuda:0").to(torch.bfloat16)
    cu = [0, 130, 207]
    want = W.packed(_host(q), _host(k), _host(v), cu, cu, 0.125, window, sinks, "bfloat16",
                    _host(do), _host(out))
    for name, t in (("out", out), ("dq", dq), ("dk", dk), ("dv", dv)):
        assert (np.abs(_host(t) - want[name][0]) <= want[name][1]).all(), name
