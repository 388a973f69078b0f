"""Large scores over the cache of 8 bits: a value's exponent keeps its bits beside them."""
import numpy as np
import pytest

import attn_window_oracle as W
from paper_2609_11938_amd import attn
from test_gpu_attn import DEV, _dt, _host, _ints, _torch
from test_gpu_attn_scaled import _empty, _np, _table

pytestmark = pytest.mark.gpu

# Scores in binary digits, below a power of two: with a value's exponent added to them
# they have one bit fewer after the point.
SCORES = [2.0 ** 7 - 2.7183, 2.0 ** 14 - 2.7183, 2.0 ** 17 - 2.7183]
LOG2E = 1.4426950408889634


def _case(lens, d, page, block, dtype, digits, sign):
    """Keys of one value each, so that every score of a sequence is the same number; values
    of any code, blocks of different scales. (arguments of the call, its scale, the values
    of each sequence's tokens)"""
    torch = _torch()
    print(f"case scores lens={lens} d={d} page={page} block={block} {dtype} {digits} {sign}",
          flush=True)
    rng = np.random.default_rng([sum(lens), d, page, block, int(digits)])
    table, pages = _table(rng, lens, page)
    codes, scales, _ = _empty(pages, page, block, 1, d)
    codes[0] = 0x38  # 1
    scales[0] = 127 + 7
    c = rng.integers(0, 256, codes[1].shape).astype(np.uint8)
    codes[1] = torch.from_numpy(np.where(c & 127 == 127, 0x38, c)).to(DEV)
    scales[1] = torch.from_numpy(rng.integers(121, 133, scales[1].shape).astype(np.uint8)).to(DEV)
    q = torch.full((len(lens), 2, d), 1.5, dtype=_dt(dtype), device=DEV)
    q[:, 1] = 0.75
    values = []
    for b, n in enumerate(lens):
        t = np.arange(n)
        x = table[b, t // page]
        values.append(W.values_of(_np(codes[1])[x, t % page, 0],
                                  _np(scales[1])[x, t % page // block, 0]))
    scale = sign * digits / LOG2E / (d * 1.5 * 2 ** 7)
    return (q, *codes, *scales, _ints(table), _ints(lens)), scale, values


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("d,page,block", [(64, 16, 16), (128, 32, 16), (64, 16, 8), (128, 8, 2)])
@pytest.mark.parametrize("digits", SCORES)
@pytest.mark.parametrize("sign", [1, -1])
def test_one_token_is_its_stored_value(d, page, block, dtype, digits, sign):
    """Alone, and as the last of many that a window of one leaves: codes have 4 bits, so
    that the stored value is one of the outputs' type."""
    args, scale, values = _case([1, 40, 700], d, page, block, dtype, digits, sign)
    out, _ = attn.opattr_attn_paged_scaled(*args, window=1, scale=scale)
    for b, v in enumerate(values):
        for head in range(2):
            np.testing.assert_array_equal(_host(out[b, head]), v[-1], err_msg=f"{b}, {head}")


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("d,page,block", [(64, 16, 16), (128, 32, 16), (64, 16, 8), (128, 8, 2)])
@pytest.mark.parametrize("digits", SCORES)
def test_equal_scores_give_the_mean(d, page, block, dtype, digits):
    """Tokens with the same score weigh the same, 1 over their number, in one tile, over the
    waves and over shares. A weight is 2^(kShift + e - n), e and n whole numbers, e within 12
    of the largest: exact in 16 bits. So the values' sum has float32's roundings alone, at
    most one a token and 2^-24 of what is added; a share's and a wave's factor and the
    quotient three more of 2^-22 (an exponential, a reciprocal, a product), and the result one
    of 16 bits."""
    u, tiny = W.UNIT[dtype], W.TINY[dtype]
    args, scale, values = _case([2, 33, 700, 4001], d, page, block, dtype, digits, 1)
    out, lse = attn.opattr_attn_paged_scaled(*args, scale=scale)
    x = digits / LOG2E
    for b, v in enumerate(values):
        n, mean, size = len(v), v.mean(0), np.abs(v).mean(0)
        for head in range(2):
            more = (n * 2.0 ** -24 + 3 * 2.0 ** -22) * size
            off = np.abs(_host(out[b, head]) - mean)
            bound = u * (np.abs(mean) + more) + more + tiny
            assert (off <= bound).all(), (b, head, off.max())
            want = x / (1 + head) + np.log(n)
            # the score's two products, the sum and its product with ln 2: 2^-24 each
            assert abs(float(lse[head, b]) - want) <= 2.0 ** -21 * abs(want) + 2.0 ** -20
