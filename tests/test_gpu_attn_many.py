"""The attention operators over more sequences than a wave has lanes, and in the
forms that only many blocks or long rows take: the same oracle and bounds as
test_gpu_attn.py."""
import numpy as np
import pytest

from paper_2609_11938_amd import attn, opattr
from test_gpu_attn import (DEV, _cache, _check_paged, _check_prompt, _cu, _ints, _prompt, _rand,
                           _torch)

pytestmark = pytest.mark.gpu


def _many(n, seed, longest):
    """n lengths: empty, short and, on both sides of every 64th, long ones."""
    rng = np.random.default_rng([n, seed])
    lens = [int(x) for x in rng.integers(0, 9, n)]
    for at in (1, 63, 64, 65, 127, 128, n - 1):
        if at < n:
            lens[at] = int(rng.integers(longest // 2, longest + 1))
    lens[2] = lens[62] = 0
    return lens


@pytest.mark.parametrize("n", [65, 128, 130])
@pytest.mark.parametrize("causal,dtype,d", [(True, "bfloat16", 64), (False, "bfloat16", 128),
                                            (True, "float16", 128), (False, "float16", 40)])
def test_prompt_many_sequences(n, causal, dtype, d):
    lens_q = _many(n, 1, 300)
    lens_k = [x + (b % 3) * 5 for b, x in enumerate(lens_q)]
    lens_k[5] = 0
    _check_prompt(_prompt(lens_q, lens_k, 4, 2, d, causal, dtype))


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype,d", [("bfloat16", 64), ("float16", 128)])
def test_prompt_many_sequences_with_split_key_tiles(dtype, d, causal):
    """Key tiles shared by blocks, more than 64 sequences: a sequence's rows come to
    more than 16 steps of 32 queries and the tiles to fewer than 192."""
    lens = [int(x) for x in np.random.default_rng(3).integers(100, 260, 67)]
    lens[0], lens[64], lens[66] = 400, 390, 300
    h = 8
    assert (sum(lens) // 128 + len(lens)) <= 192 and sum(lens) * h // 32 // len(lens) >= 24
    _check_prompt(_prompt(lens, lens, h, 1, d, causal, dtype))


@pytest.mark.parametrize("causal,d", [(True, 16), (False, 16), (True, 72)])
def test_prompt_key_tiles_split_by_long_runs(causal, d):
    """Key tiles of so many heads that every unit has a block: split by 24 steps."""
    lens, g, group = [470, 330], 25, 4
    assert (sum(lens) // 128 + 2) * g > 192 and sum(lens) * group // 32 // 2 >= 2 * 24
    _check_prompt(_prompt(lens, lens, g * group, g, d, causal, "bfloat16"))


@pytest.mark.parametrize("lens", [([900], [900]), ([1, 300], [1700, 900]), ([800], [780])], ids=str)
@pytest.mark.parametrize("dtype,d", [("bfloat16", 64), ("float16", 128)])
def test_prompt_two_groups_without_a_mask(lens, dtype, d):
    """Many keys to a few rows, every key seen."""
    _check_prompt(_prompt(*lens, 2, 1, d, False, dtype))


@pytest.mark.parametrize("n", [65, 130])
@pytest.mark.parametrize("h,g,d,dtype", [(4, 2, 64, "bfloat16"), (8, 1, 128, "float16")])
def test_paged_many_sequences(n, h, g, d, dtype):
    """Sequences of several shares on both sides of every 64th."""
    _check_paged(_many(n, 2, 1100), h, g, d, 16, dtype)


@pytest.mark.parametrize("n", [64, 65, 130, 200])
def test_append_many_sequences(n):
    torch = _torch()
    rng = np.random.default_rng(n)
    g, d, page = 3, 40, 8
    before = [int(x) for x in rng.integers(0, 20, n)]
    new = [int(x) for x in rng.integers(0, 7, n)]
    new[0] = new[62] = 0
    new[-1], new[63] = 11, 9
    total = [x + y for x, y in zip(before, new)]
    cache, table, _ = _cache(rng, [0] * n, g, d, page, "bfloat16", extra=sum(
        -(-t // page) for t in total) + 3, width=max(total) // page + 2)
    ids = rng.permutation(cache.shape[1])
    at = 0
    for b, t in enumerate(total):
        c = -(-t // page)
        table[b, :c] = ids[at:at + c]
        at += c
    cache.fill_(-1)
    k, _ = _rand(rng, (sum(new), g, d), "bfloat16")
    v, _ = _rand(rng, (sum(new), g, d), "bfloat16")
    diag = attn.new_diag(DEV)
    print(f"case append of {n} sequences", flush=True)
    after = attn.opattr_kv_append(k, v, _ints(_cu(new)), cache[0], cache[1], _ints(table),
                                  _ints(before), diag=diag)
    assert after.tolist() == total and opattr.read_diag(diag)["status"] == 0
    row = np.repeat(np.arange(n), new)
    pos = np.concatenate([b + np.arange(c) for b, c in zip(before, new)]).astype(np.int64)
    where = torch.from_numpy(table[row, pos // page]).to(DEV)
    slot = torch.from_numpy(pos % page).to(DEV)
    want = torch.full_like(cache, -1)
    want[0][where, slot], want[1][where, slot] = k, v
    assert torch.equal(cache, want)
