"""The workspace of the window attention's gradient from above (no GPU): a few sinks cost
what their own partial results take, whatever the key heads and the sequences' number."""
import pytest

from test_attn_abi import _shape, lib  # noqa: F401 (a fixture)

# tokens, sequences, query and key heads, head_dim, window
SHAPES = [(48000, 32, 32, 8, 128, 512), (48000, 32, 32, 32, 128, 512), (6000, 32, 32, 32, 128, 64),
          (8192, 16, 32, 32, 128, 64), (100_000, 1, 16, 4, 128, 1024), (20_000, 300, 8, 8, 64, 50),
          (500_000, 1000, 64, 8, 128, 400), (30_000, 12, 12, 12, 64, 128)]


def _extra(lib, shape, sinks):  # noqa: F811
    n, seqs, h, g, d, window = shape
    a = _shape(n_q=n, n_k=n, n_seqs=seqs, n_heads=h, n_kv_heads=g, head_dim=d)
    need = lib.opattr_attn_prompt_window_grad_workspace_bytes
    return need(a, window, sinks) - need(a, window, 0)


@pytest.mark.parametrize("sinks", [1, 4, 128])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_sinks_of_one_key_tile(lib, shape, sinks):  # noqa: F811
    """A tile's block takes 32 steps of 32 queries and leaves dk and dv of 128 keys in
    float32: 4 head_dim 2 128 bytes for 1024 rows of 2 head_dim bytes, half of the queries'
    own bytes; twice that where a sequence's last block has few steps, and what the last
    rows of its last tile add to it."""
    n, _, h, _, d, _ = shape
    assert _extra(lib, shape, sinks) <= 1.25 * 2 * n * h * d


@pytest.mark.parametrize("sinks", [129, 300, 8192, 1 << 29])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_sinks_of_many_key_tiles(lib, shape, sinks):  # noqa: F811
    """2048 blocks of all key heads are shared tiles' at most, twice that where a
    sequence's last block has few steps."""
    g, d = shape[3:5]
    assert _extra(lib, shape, sinks) <= 2 * (2048 + g) * 128 * 2 * d * 4


@pytest.mark.parametrize("n", [4000, 1 << 18])
def test_more_key_heads_than_shared_blocks(lib, n):  # noqa: F811
    """No tile is shared then."""
    a = _shape(n_q=n, n_k=1000, n_seqs=2, n_heads=4096, n_kv_heads=4096, head_dim=64)
    need = lib.opattr_attn_prompt_window_grad_workspace_bytes
    assert need(a, 50, 0) > 0
    assert all(need(a, 50, sinks) == need(a, 50, 0) for sinks in (1, 200, 1 << 29))
