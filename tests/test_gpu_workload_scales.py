"""The bytes that the workload records for attention over a cache of 8 bits: its codes, its
exponents and the queries."""
import numpy as np
import pytest

import attn_window_oracle as W

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("window,sinks", [(None, 0), (20, 3), (20, 9), (1, 0), (3, 40), (500, 2)])
def test_recorded_bytes_have_the_exponents(window, sinks):
    from paper_2609_11938_amd import workload

    lens, page, kv, d, heads = (50, 9, 33), 8, 2, 64, 4
    rec = workload.Recorder()
    workload.serve(rec, lens=lens, steps=3, layers=1, heads=heads, kv_heads=kv, head_dim=d,
                   page_size=page, window=window, sinks=sinks, scaled=True)
    tr = rec.trace()
    at = np.flatnonzero(tr["name_id"] == rec.names.index("attn_paged_scaled"))
    for step in range(3):
        want = 0
        for n in lens:
            n += step + 1
            seen = W.visible(1, n, window or n, sinks)[0]
            want += 2 * kv * (d * seen.sum() + len(np.unique(np.flatnonzero(seen) // page)))
        want += 3 * heads * d * 2
        assert tr["counters"][at[step], workload.READ] == want
