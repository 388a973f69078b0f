"""The paged cache of 8 bits on the GPU against the 64-bit oracle
(tests/attn_window_oracle.py): appends bit for bit, attention within its bounds, at
the blocks, scales, sizes and layouts where they can go wrong."""
import math

import numpy as np
import pytest

import attn_window_oracle as W
from paper_2609_11938_amd import attn, opattr
from test_gpu_attn import DATA, DEV, _cu, _dt, _host, _ints, _rand, _torch, _within

pytestmark = pytest.mark.gpu


def _empty(pages, page, block, g, d, order="nhd", fill=0x7f, scale=255):
    """codes [2, pages, page, g, d] and scales [2, pages, blocks, g] that hold NaN."""
    torch = _torch()
    like = dict(dtype=torch.uint8, device=DEV)
    if order == "nhd":
        codes = torch.full((2, pages, page, g, d), fill, **like)
    elif order == "hnd":
        codes = torch.full((2, pages, g, page, d), fill, **like).transpose(2, 3)
    else:  # a page's scales behind its codes
        each = page * g * d
        room = -(-(page // block) * g // 16) * 16
        pool = torch.full((2, pages, each + room), fill, **like)
        scales = pool[:, :, each:each + page // block * g].view(2, pages, page // block, g)
        scales.fill_(scale)
        return pool[:, :, :each].view(2, pages, page, g, d), scales, pool
    return codes, torch.full((2, pages, page // block, g), scale, **like), None


def _table(rng, lens, page, extra=3, width=None):
    counts = [-(-n // page) for n in lens]
    pages = sum(counts) + extra
    width = max(counts, default=0) + 1 if width is None else width
    ids = rng.permutation(pages)
    table = np.full((len(lens), width), -1, np.int64)
    at = 0
    for b, n in enumerate(counts):
        table[b, :n] = ids[at:at + n]
        at += n
    return table, pages


def _np(t):
    return t.cpu().numpy()


def _same_codes(got, want, name):
    """Equal, NaN of either sign for NaN."""
    got, want = _np(got), np.asarray(want)
    off = (got != want) & ~((got & 127 == 127) & (want & 127 == 127))
    assert not off.any(), f"{name}: {int(off.sum())} codes differ, first at {np.argwhere(off)[0]}"


def _append(codes, scales, new, cu, table, lens, bad=0):
    """opattr_kv_append_scaled, checked against the oracle; returns the new lengths."""
    torch = _torch()
    before = [(_np(codes[i]).copy(), _np(scales[i]).copy()) for i in range(2)]
    diag = attn.new_diag(DEV)
    after = attn.opattr_kv_append_scaled(new[0], new[1], _ints(cu), codes[0], codes[1], scales[0],
                                         scales[1], _ints(table), _ints(lens), diag=diag)
    torch.cuda.synchronize()
    for i, name in enumerate("kv"):
        c, s, n = W.append_scaled(*before[i], _host(new[i]), cu, table, lens)
        _same_codes(codes[i], c, name)
        np.testing.assert_array_equal(_np(scales[i]), s, err_msg=f"{name} scales")
        assert n == bad
    d = opattr.read_diag(diag)
    assert d["status"] == (DATA if bad else 0) and d["bad_records"] == bad
    return after.tolist()


def _rows(rng, n, g, d, dtype, spread=3.0):
    """Keys and values, slices of wider rows, whose heads, channels and tokens differ in
    size by powers of two."""
    torch = _torch()
    x = rng.normal(size=(n, 2 * g + 1, d)) * 2.0 ** (spread * rng.normal(size=(n, 2 * g + 1, 1))) * \
        2.0 ** (spread * rng.normal(size=(1, 2 * g + 1, d)) / 2)
    x = np.clip(x, -6e4, 6e4)
    rows = torch.from_numpy(x.astype(np.float32)).to(DEV, _dt(dtype))
    return rows[:, :g], rows[:, g:2 * g]


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("order", ["nhd", "hnd", "pool"])
@pytest.mark.parametrize("g,d,page,block", [(2, 64, 16, 16), (3, 48, 8, 4), (1, 128, 1, 1),
                                            (12, 64, 32, 32), (2, 128, 64, 16), (1, 16, 1024, 512),
                                            (2, 128, 128, 128), (5, 112, 16, 2)])
def test_append_in_parts(g, d, page, block, order, dtype):
    """Prompts, then parts that begin inside blocks, then single tokens: each append as
    the definition has it, on what the ones before left."""
    rng = np.random.default_rng([g, d, page, block])
    parts = [[7, 0, 33, 40, 1], [5, 1, 0, 17, 1], [1, 1, 1, 1, 1], [1, 1, 1, 0, 1], [30, 2, 19, 64, 1]]
    total = np.sum(parts, axis=0)
    table, pages = _table(rng, total, page)
    codes, scales, _ = _empty(pages, page, block, g, d, order)
    lens = [0] * 5
    for turn, new in enumerate(parts):
        print(f"case append g={g} d={d} page={page} block={block} {order} {dtype} part {turn}",
              flush=True)
        rows = _rows(rng, sum(new), g, d, dtype)
        lens = _append(codes, scales, rows, _cu(new), table, lens)
    assert lens == total.tolist()


@pytest.mark.parametrize("n", [64, 65, 130])
def test_append_many_sequences(n):
    rng = np.random.default_rng(n)
    before = [int(x) for x in rng.integers(0, 20, n)]
    new = [int(x) for x in rng.integers(0, 7, n)]
    new[0] = new[62] = 0
    new[-1], new[63] = 31, 50
    table, pages = _table(rng, np.add(before, new), 8)
    codes, scales, _ = _empty(pages, 8, 4, 3, 32)
    lens = _append(codes, scales, _rows(rng, sum(before), 3, 32, "bfloat16"), _cu(before), table,
                   [0] * n)
    _append(codes, scales, _rows(rng, sum(new), 3, 32, "bfloat16"), _cu(new), table, lens)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
def test_append_every_value(dtype):
    """Every value of the type beside a block's largest: the codes are the nearest, ties
    to even, at scales from the smallest to the largest."""
    torch = _torch()
    bits = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16).view(_dt(dtype)).to(DEV)
    rows = bits.view(512, 1, 128)
    table, pages = _table(np.random.default_rng(0), [512], 1)
    codes, scales, _ = _empty(pages, 1, 1, 1, 128)
    _append(codes, scales, (rows, rows.flip(2)), [0, 512], table, [0])
    for top in (1.0, 448.0, 449.0, 0.875, 0.8751, 2.0 ** -14, 3e4):
        x = bits[bits.float().abs() <= top].reshape(-1)
        x = torch.cat((x, x.new_full((-x.numel() % 127,), 0.0))).view(-1, 127)
        x = torch.cat((x, x.new_full((x.shape[0], 1), top)), 1)[:, None]
        pick = torch.arange(0, x.shape[0], 7)
        table, pages = _table(np.random.default_rng(0), [len(pick)], 1)
        codes, scales, _ = _empty(pages, 1, 1, 1, 128)
        _append(codes, scales, (x[pick], -x[pick]), [0, len(pick)], table, [0])


def test_append_blocks_grow():
    """Tokens 2^10 larger than those before in their block, one by one: what is there
    goes over to the new exponent; zeros, infinities and NaN have no part in it."""
    torch = _torch()
    rng = np.random.default_rng(3)
    table, pages = _table(rng, [16, 16], 16)
    codes, scales, _ = _empty(pages, 16, 16, 2, 32)
    lens = [0, 0]
    for t in range(16):
        x = rng.normal(size=(2, 2, 2, 32)) * 2.0 ** ((t - 8) * (10 if t % 3 else 1))
        if t in (0, 5):
            x[:] = 0
        new = torch.from_numpy(x.astype(np.float32)).to(DEV, torch.bfloat16)
        if t in (2, 9):
            new[0, 0, :, 3] = float("inf")
            new[1, 1, 1, 4] = float("nan")
            new[1, 0, 0] = -float("inf")
        lens = _append(codes, scales, new, [0, 1, 2], table, lens)


def test_append_out_of_place_is_flagged():
    rng = np.random.default_rng(9)
    table, pages = _table(rng, [20, 20, 20], 16, width=2)
    codes, scales, _ = _empty(pages, 16, 8, 2, 64)
    rows = _rows(rng, 45, 2, 64, "bfloat16")
    bad = table.copy()
    bad[0, 1], bad[2, 0] = 5000, -2
    _append(codes, scales, rows, [0, 20, 30, 45], bad, [0, 27, -6], bad=4 + 5 + 6 + 9)
    codes, scales, _ = _empty(pages, 16, 8, 2, 64)
    _append(codes, scales, rows, [0, 20, 30, 45], table, [-3, 2 ** 31 - 5, 100], bad=3 + 10 + 15)


def test_append_offsets_are_clamped_and_flagged():
    torch = _torch()
    rng = np.random.default_rng(9)
    table, pages = _table(rng, [40, 40], 16)
    rows = _rows(rng, 30, 2, 64, "bfloat16")
    for cu in ([0, 10, 99], [-5, 10, 30], [0, 25, 20]):
        codes, scales, _ = _empty(pages, 16, 8, 2, 64)
        diag = attn.new_diag(DEV)
        attn.opattr_kv_append_scaled(*rows, _ints(cu), *codes, *scales, _ints(table), _ints([0, 0]),
                                     diag=diag)
        torch.cuda.synchronize()
        assert opattr.read_diag(diag)["status"] == DATA


def test_append_nothing():
    torch = _torch()
    rng = np.random.default_rng(1)
    table, pages = _table(rng, [5], 16)
    codes, scales, _ = _empty(pages, 16, 16, 2, 64)
    z = torch.zeros(0, 2, 64, dtype=torch.float16, device=DEV)
    assert _append(codes, scales, (z, z), [0, 0], table, [3]) == [3]


# --------------------------------------------------------------------------- #
# attention                                                                   #
# --------------------------------------------------------------------------- #


def _filled(rng, lens, g, d, page, block, dtype, order="nhd", spread=2.0):
    """A cache with the sequences' tokens, its unused places NaN."""
    table, pages = _table(rng, lens, page)
    codes, scales, pool = _empty(pages, page, block, g, d, order)
    if sum(lens):
        rows = _rows(rng, sum(lens), g, d, dtype, spread)
        attn.opattr_kv_append_scaled(*rows, _ints(_cu(lens)), *codes, *scales, _ints(table),
                                     _ints([0] * len(lens)))
    return codes, scales, table, pool


def _tokens(codes, scales, table, b, n, j):
    """Head j's codes and exponents' bytes of sequence b's tokens."""
    page, block = codes.shape[2], codes.shape[2] // scales.shape[2]
    t = np.arange(n)
    x = table[b, t // page]
    return [(_np(codes[i])[x, t % page, j], _np(scales[i])[x, t % page // block, j])
            for i in range(2)]


def _check(codes, scales, table, lens, q, window=None, sinks=0, scale=None, ws=None, diag=True,
           status=0):
    torch = _torch()
    h, d = q.shape[1:]
    g = codes.shape[3]
    dtype = str(q.dtype).split(".")[1]
    scale = 1 / math.sqrt(d) if scale is None else scale
    rec = attn.new_diag(DEV) if diag else None
    args = (q, *codes, *scales, _ints(table), _ints(lens))
    kw = dict(window=window, sinks=sinks, scale=scale, ws=ws)
    out, lse = attn.opattr_attn_paged_scaled(*args, diag=rec, **kw)
    torch.cuda.synchronize()
    qh = _host(q)
    host = _np(codes), _np(scales)
    for b, n in enumerate(lens):
        seen = W.visible(1, n, window or 1 << 30, sinks)[0]
        page, block = codes.shape[2], codes.shape[2] // scales.shape[2]
        t = np.arange(n)
        x = table[b, t // page]
        for j in range(h):
            k, v = ((host[0][i][x, t % page, j * g // h],
                     host[1][i][x, t % page // block, j * g // h]) for i in range(2))
            o, s = W.head_scaled(qh[b, j], *k, *v, scale, seen, dtype)
            _within(out[b, j], o, f"out[{b}, {j}]")
            _within(lse[j, b], s, f"lse[{j}, {b}]")
    if diag:
        assert opattr.read_diag(rec)["status"] == status
    again, _ = attn.opattr_attn_paged_scaled(*args, **kw)
    assert torch.equal(out, again), "runs differ"
    return out, lse


def _case(lens, h, g, d, page, block, dtype, order="nhd", window=None, sinks=0, ws=None, spread=2.0):
    print(f"case scaled lens={lens} heads={h}/{g} d={d} page={page} block={block} {dtype} {order} "
          f"window={window} sinks={sinks}", flush=True)
    rng = np.random.default_rng([h, g, d, page, block, len(lens)])
    codes, scales, table, _ = _filled(rng, lens, g, d, page, block, dtype, order, spread)
    q, _ = _rand(rng, (len(lens), h, d), dtype, 0.2)
    return _check(codes, scales, table, lens, q, window, sinks, ws=ws)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("h,g,d,page,block", [
    (2, 2, 64, 16, 16), (8, 2, 128, 16, 4), (16, 1, 128, 32, 32), (3, 1, 80, 1, 1),
    (4, 4, 16, 64, 16), (12, 12, 64, 4, 2), (5, 1, 96, 128, 64), (2, 1, 48, 1024, 512)])
def test_scaled_heads(h, g, d, page, block, dtype):
    _case([1, 37, 0, 130], h, g, d, page, block, dtype)


@pytest.mark.parametrize("lens", [[0], [1], [31], [32], [33], [255], [256], [257], [1025], [0, 0],
                                  [5000, 3, 0, 700], [1] * 70], ids=lambda v: str(v)[:30])
def test_scaled_lengths(lens):
    _case(lens, 4, 1, 64, 16, 16, "bfloat16")


@pytest.mark.parametrize("order", ["hnd", "pool"])
def test_scaled_layouts(order):
    _case([100, 45], 4, 2, 64, 16, 8, "bfloat16", order)


def test_scaled_long_split():
    """One sequence over many shares, beside short ones; the workspace holds another
    call's partial results."""
    ws = attn.Workspace(DEV)
    _case([40000], 4, 2, 64, 16, 16, "float16", ws=ws)
    _case([20011, 1, 0, 300], 8, 2, 128, 64, 64, "bfloat16", ws=ws)


@pytest.mark.parametrize("n", [65, 130])
def test_scaled_many_sequences(n):
    rng = np.random.default_rng(n)
    lens = [int(x) for x in rng.integers(0, 9, n)]
    for at in (1, 63, 64, n - 1):
        lens[at] = int(rng.integers(400, 1100))
    _case(lens, 4, 2, 64, 16, 16, "bfloat16")


@pytest.mark.parametrize("window,sinks", [(1, 0), (31, 1), (32, 0), (100, 4), (252, 4), (600, 300),
                                          (5, 1000)])
@pytest.mark.parametrize("dtype,d,page,block", [("bfloat16", 64, 16, 8), ("float16", 128, 16, 8),
                                                ("bfloat16", 128, 16, 16),
                                                ("float16", 64, 64, 32)])
def test_scaled_window(window, sinks, dtype, d, page, block):
    _case([5000, 3, 0, 700, 256, 257], 4, 1, d, page, block, dtype, window=window, sinks=sinks)


@pytest.mark.parametrize("sinks", [0, 1, 15, 16, 17, 31, 33, 128, 130])
@pytest.mark.parametrize("window", [1, 15, 16, 17, 100, 113])
def test_scaled_window_edges(window, sinks):
    """Sinks and windows that end and begin on, before and after a run of 16 tokens and a
    tile of 32, for lengths on both sides of them."""
    lens = [window + sinks + n for n in (-1, 0, 1, 14, 15, 16, 17, 31, 33, 300)]
    _case(lens, 2, 1, 64, 32, 16, "bfloat16", window=window, sinks=sinks)


def test_scaled_window_leaves_pages_behind():
    """Entries of pages of which no token is seen say nothing, their codes neither."""
    torch = _torch()
    rng = np.random.default_rng(21)
    lens, page, window, sinks = [500, 90, 1300], 16, 75, 20
    codes, scales, table, _ = _filled(rng, lens, 2, 64, page, 16, "bfloat16")
    q, _ = _rand(rng, (3, 4, 64), "bfloat16", 0.2)
    want, wl = _check(codes, scales, table, lens, q, window, sinks)
    for b, n in enumerate(lens):
        for x in range(-(-n // page)):
            if x * page >= sinks and (x + 1) * page <= n - window:
                codes[:, table[b, x]] = 0x7f
                scales[:, table[b, x]] = 255
                table[b, x] = (-1, 1 << 30, table[b, x])[x % 3]
    diag = attn.new_diag(DEV)
    out, lse = attn.opattr_attn_paged_scaled(q, *codes, *scales, _ints(table), _ints(lens),
                                             window=window, sinks=sinks, diag=diag)
    assert torch.equal(out, want) and torch.equal(lse, wl)
    assert opattr.read_diag(diag)["status"] == 0


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("spread", [0.0, 5.0])
@pytest.mark.parametrize("block", [4, 16])
def test_scaled_blocks_of_other_sizes(dtype, spread, block):
    """Blocks whose scales differ by many powers of two, in one tile and over shares:
    the weights keep their bits where the scale is small and where it is large."""
    torch = _torch()
    rng = np.random.default_rng(11)
    lens, g, d = [900, 70], 2, 64
    codes, scales, table, _ = _filled(rng, lens, g, d, 16, block, dtype, spread=0.5)
    # a token's key and value scales, one against the other; large values with little weight
    shift = torch.from_numpy(np.round(spread * 4 * rng.normal(size=scales[1].shape)).clip(-40, 40)
                             ).to(DEV)
    scales[1] = (scales[1].double() + shift).clamp(0, 254).to(torch.uint8)
    scales[1][codes.shape[1] // 2:] = 3
    q, _ = _rand(rng, (2, 4, d), dtype, 0.5)
    if dtype == "float16":  # values stay in float16
        scales[1] = scales[1].clamp(max=127 + 6)
    _check(codes, scales, table, lens, q)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("block", [8, 16])
def test_scaled_largest_and_smallest_scales(dtype, block):
    """Values near the type's largest, and down to the smallest exponent."""
    torch = _torch()
    rng = np.random.default_rng(12)
    lens, g, d = [300, 40], 1, 64
    for e in (127 + (118 if dtype == "bfloat16" else 6), 20, 1, 0):
        codes, scales, table, _ = _filled(rng, lens, g, d, 16, block, dtype, spread=0.0)
        codes.bitwise_and_(0xf7)  # no NaN, at most 240
        scales[1].fill_(e)
        q, _ = _rand(rng, (2, 2, d), dtype)
        _check(codes, scales, table, lens, q)


@pytest.mark.parametrize("block", [8, 16])
def test_scaled_nan_codes_and_scales(block):
    """A NaN code or scale of a key makes its sequence's heads NaN, of a value the
    outputs that it meets; of a token that is not seen, nothing."""
    torch = _torch()
    rng = np.random.default_rng(13)
    lens, g, d, page = [100, 60], 2, 64, 16
    codes, scales, table, _ = _filled(rng, lens, g, d, page, block, "bfloat16")
    q, _ = _rand(rng, (2, 4, d), "bfloat16")
    args = (_ints(table), _ints(lens))
    want, wl = attn.opattr_attn_paged_scaled(q, *codes, *scales, *args)
    x, slot = int(table[0, 2]), 5  # token 37

    def got(**kw):
        return attn.opattr_attn_paged_scaled(q, *codes, *scales, *args, **kw)

    def others(out, lse, heads):
        rest = [j for j in range(4) if j not in heads]
        assert torch.equal(out[1], want[1]) and torch.equal(lse[:, 1], wl[:, 1])
        assert torch.equal(out[0, rest], want[0, rest]) and torch.equal(lse[rest, 0], wl[rest, 0])

    old = int(codes[0, x, slot, 1, 9])
    codes[0, x, slot, 1, 9] = 0xff
    out, lse = got()
    assert torch.isnan(out[0, 2:]).all() and torch.isnan(lse[2:, 0]).all()
    others(out, lse, (2, 3))
    out, lse = got(window=62, sinks=37)  # the token is the first that is not seen
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
    codes[0, x, slot, 1, 9] = old
    old = int(codes[1, x, slot, 0, 3])
    codes[1, x, slot, 0, 3] = 0x7f
    out, lse = got()
    assert torch.isnan(out[0, :2, 3]).all() and torch.equal(lse, wl)
    keep = [c for c in range(d) if c != 3]
    assert torch.equal(out[0, :2][:, keep], want[0, :2][:, keep])
    others(out, lse, (0, 1))
    codes[1, x, slot, 0, 3] = old
    for i in range(2):
        was = int(scales[i, x, 0, 0])
        scales[i, x, 0, 0] = 255
        out, lse = got()
        assert torch.isnan(out[0, :2]).all()
        assert torch.isnan(lse[:2, 0]).all() if i == 0 else torch.equal(lse, wl)
        others(out, lse, (0, 1))
        out, lse = got(window=52, sinks=32)
        assert torch.isfinite(out).all()
        scales[i, x, 0, 0] = was


@pytest.mark.parametrize("block", [8, 16])
def test_scaled_bad_table_and_lens(block):
    torch = _torch()
    rng = np.random.default_rng(5)
    lens, page = [50, 40], 16
    codes, scales, table, _ = _filled(rng, lens, 2, 64, page, block, "bfloat16")
    q, _ = _rand(rng, (2, 4, 64), "bfloat16")
    for where, value in (((0, 1), 10_000), ((1, 0), -3)):
        bad = table.copy()
        bad[where] = value
        diag = attn.new_diag(DEV)
        out, lse = attn.opattr_attn_paged_scaled(q, *codes, *scales, _ints(bad), _ints(lens),
                                                 diag=diag)
        torch.cuda.synchronize()
        d = opattr.read_diag(diag)
        assert d["status"] == DATA and d["bad_records"] == page
        b, x = where
        seen = np.ones(lens[b], bool)
        seen[x * page:(x + 1) * page] = False
        k, v = _tokens(codes, scales, table, b, lens[b], 0)
        o, s = W.head_scaled(_host(q)[b, 0], *k, *v, 0.125, seen, "bfloat16")
        _within(out[b, 0], o, "out")
        _within(lse[0, b], s, "lse")
    for window, sinks in ((20, 4), (20, 18), (24, 4), (2, 50)):
        bad = table.copy()  # tokens 16 to 31 of the first
        bad[0, 1] = -1
        diag = attn.new_diag(DEV)
        out, lse = attn.opattr_attn_paged_scaled(q, *codes, *scales, _ints(bad), _ints(lens),
                                                 window=window, sinks=sinks, diag=diag)
        torch.cuda.synchronize()
        seen = W.visible(1, lens[0], window, sinks)[0]
        assert opattr.read_diag(diag)["bad_records"] == seen[16:32].sum() > 0
        seen[16:32] = False
        k, v = _tokens(codes, scales, table, 0, lens[0], 0)
        o, s = W.head_scaled(_host(q)[0, 0], *k, *v, 0.125, seen, "bfloat16")
        _within(out[0, 0], o, "out")
        _within(lse[0, 0], s, "lse")
    codes.fill_(0x38)
    scales.fill_(127)
    full = _ints(rng.permutation(codes.shape[1])[:8].reshape(2, 4))
    want, _ = attn.opattr_attn_paged_scaled(q, *codes, *scales, full, _ints([64, 0]))
    diag = attn.new_diag(DEV)
    got, _ = attn.opattr_attn_paged_scaled(q, *codes, *scales, full, _ints([9999, -7]), diag=diag)
    assert torch.equal(got, want) and opattr.read_diag(diag)["status"] == DATA


def test_scaled_offsets_past_32_bits():
    """Pages beyond 2^32 bytes from the first."""
    torch = _torch()
    rng = np.random.default_rng(6)
    page, g, d = 64, 8, 128
    pages = (1 << 32) // (page * g * d) + 40
    codes = torch.zeros(2, pages, page, g, d, dtype=torch.uint8, device=DEV)
    scales = torch.zeros(2, pages, 4, g, dtype=torch.uint8, device=DEV)
    n = 3 * page - 5
    table = np.array([[pages - 1, 3, pages - 2]])
    k, v = _rows(rng, n, g, d, "bfloat16")
    attn.opattr_kv_append_scaled(k, v, _ints([0, n]), *codes, *scales, _ints(table), _ints([0]))
    near = [x.index_select(1, torch.tensor([3, pages - 2, pages - 1], device=DEV)).contiguous()
            for x in (codes, scales)]
    small = np.array([[2, 0, 1]])
    c2, s2 = torch.zeros_like(near[0]), torch.zeros_like(near[1])
    attn.opattr_kv_append_scaled(k, v, _ints([0, n]), *c2, *s2, _ints(small), _ints([0]))
    assert torch.equal(c2, near[0]) and torch.equal(s2, near[1])
    q, _ = _rand(rng, (1, 8, d), "bfloat16", 0.2)
    got = attn.opattr_attn_paged_scaled(q, *codes, *scales, _ints(table), _ints([n]))
    want = attn.opattr_attn_paged_scaled(q, *c2, *s2, _ints(small), _ints([n]))
    assert all(torch.equal(x, y) for x, y in zip(got, want))


def test_scaled_types_of_the_cache():
    """float8_e4m3fn codes and float8_e8m0fnu exponents are the same bytes."""
    torch = _torch()
    rng = np.random.default_rng(14)
    lens = [70]
    codes, scales, table, _ = _filled(rng, lens, 1, 64, 16, 16, "bfloat16")
    c2, s2 = torch.zeros_like(codes), torch.zeros_like(scales)
    q, _ = _rand(rng, (1, 2, 64), "bfloat16")
    rows = _rows(np.random.default_rng(15), 70, 1, 64, "bfloat16")
    for c, s in ((codes, scales), (c2.view(torch.float8_e4m3fn), s2.view(torch.float8_e8m0fnu))):
        c.view(torch.uint8).zero_()
        s.view(torch.uint8).zero_()
        attn.opattr_kv_append_scaled(*rows, _ints([0, 70]), *c, *s, _ints(table), _ints([0]))
    assert torch.equal(codes, c2) and torch.equal(scales, s2)
    a = attn.opattr_attn_paged_scaled(q, *codes, *scales, _ints(table), _ints(lens))
    b = attn.opattr_attn_paged_scaled(q, *c2.view(torch.float8_e4m3fn),
                                      *s2.view(torch.float8_e8m0fnu), _ints(table), _ints(lens))
    assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_scaled_graph_replays():
    """An append and the attention captured with buffers of the caller's, replayed with
    new inputs between eager work: every replay as the eager calls."""
    torch = _torch()
    rng = np.random.default_rng(16)
    lens, g, d = [700, 33, 12], 2, 64
    total = [n + 1 for n in lens]
    table, pages = _table(rng, total, 16)
    codes, scales, _ = _empty(pages, 16, 16, g, d)
    rows = _rows(rng, sum(lens), g, d, "bfloat16")
    attn.opattr_kv_append_scaled(*rows, _ints(_cu(lens)), *codes, *scales, _ints(table),
                                 _ints([0] * 3))
    new = torch.randn(3, 8, d, device=DEV).to(torch.bfloat16)
    k, v, q = new[:, :2], new[:, 2:4], new[:, 4:]
    t, n, cu = _ints(table), _ints(lens), _ints([0, 1, 2, 3])
    after, ws = torch.empty_like(n), attn.Workspace(DEV)

    def step(c, s, **kw):
        attn.opattr_kv_append_scaled(k, v, cu, *c, *s, t, n, lens_out=after)
        return attn.opattr_attn_paged_scaled(q, *c, *s, t, after, **kw)

    start = codes.clone(), scales.clone()
    out, lse = step(codes, scales, ws=ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(codes, scales, ws=ws, out=out, lse=lse)
    for turn in range(3):
        new.mul_(1.7)
        codes.copy_(start[0])
        scales.copy_(start[1])
        c, s = codes.clone(), scales.clone()
        want, wl = step(c, s)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, wl), turn
        assert torch.equal(c, codes) and torch.equal(s, scales), turn


def test_scaled_other_stream():
    torch = _torch()
    rng = np.random.default_rng(17)
    lens = [1500, 33]
    codes, scales, table, _ = _filled(rng, lens, 2, 64, 16, 16, "float16")
    q, _ = _rand(rng, (2, 4, 64), "float16", 0.2)
    args = (q, *codes, *scales, _ints(table), _ints(lens))
    want, wl = attn.opattr_attn_paged_scaled(*args, window=300, sinks=2)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out, lse = attn.opattr_attn_paged_scaled(*args, window=300, sinks=2, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(lse, wl)


def test_append_other_stream():
    torch = _torch()
    rng = np.random.default_rng(20)
    table, pages = _table(rng, [300, 41], 16)
    rows = _rows(rng, 341, 2, 64, "bfloat16")
    args = (_ints([0, 300, 341]), _ints(table), _ints([0, 0]))
    done = []
    side = torch.cuda.Stream()
    for stream in (None, side):
        codes, scales, _ = _empty(pages, 16, 16, 2, 64)
        torch.cuda.synchronize()
        after = attn.opattr_kv_append_scaled(*rows, args[0], *codes, *scales, *args[1:],
                                             stream=stream)
        torch.cuda.synchronize()
        done.append((codes, scales, after))
    assert all(torch.equal(x, y) for x, y in zip(*done))


def test_scaled_cache_forks_and_compacts():
    """Scales behind the codes in a page's own bytes: a fork copies both, a compaction
    moves both, and the continued and forked sequences go their own ways."""
    torch = _torch()
    rng = np.random.default_rng(18)
    g, d, page, block = 2, 64, 8, 4
    table, _ = _table(rng, [20, 9], page, width=6)
    pages = 24
    codes, scales, pool = _empty(pages, page, block, g, d, "pool")
    lens, past = [20, 9], []
    rows = _rows(rng, 29, g, d, "bfloat16")
    lens = _append(codes, scales, rows, _cu(lens), table, [0, 0])
    f = attn.opattr_pages_fork(pool, page, _ints(table), _ints(lens), _ints([0, 0, 1]),
                               _ints([28, 28, 17]))
    c = attn.opattr_pages_compact(pool, f["table"])
    t2, lens = _np(c["table"]).astype(np.int64), f["lens"].tolist()
    assert lens == [20, 20, 9]
    for step in range(6):
        lens = _append(codes, scales, _rows(rng, 3, g, d, "bfloat16"), [0, 1, 2, 3], t2, lens)
    q, _ = _rand(rng, (3, 4, d), "bfloat16", 0.2)
    _check(codes, scales, t2, lens, q)
    for i in range(2):
        a, b = (_tokens(codes, scales, t2, r, 16, 0)[i] for r in (0, 1))
        assert all(np.array_equal(x, y) for x, y in zip(a, b))


def test_scaled_binding_refuses():
    torch = _torch()
    rng = np.random.default_rng(19)
    codes, scales, table, _ = _filled(rng, [20], 2, 64, 16, 8, "bfloat16")
    q, _ = _rand(rng, (1, 4, 64), "bfloat16")
    k = q[:, :2]
    t, n, cu = _ints(table), _ints([20]), _ints([0, 1])
    (kc, vc), (ks, vs) = codes, scales

    def attend(q=q, kc=kc, vc=vc, ks=ks, vs=vs, t=t, n=n, **kw):
        return attn.opattr_attn_paged_scaled(q, kc, vc, ks, vs, t, n, **kw)

    def append(k=k, v=k, cu=cu, kc=kc, vc=vc, ks=ks, vs=vs, t=t, n=n, **kw):
        return attn.opattr_kv_append_scaled(k, v, cu, kc, vc, ks, vs, t, n, **kw)

    both = [dict(kc=kc.bfloat16()), dict(kc=kc[:, :8]), dict(vc=vc[..., :48]), dict(ks=ks.float()),
            dict(ks=ks[:1]), dict(ks=ks[:, :, :1], vs=vs[:, :, :1]), dict(vs=vs.transpose(1, 2)),
            dict(kc=kc[..., :56], vc=vc[..., :56]), dict(kc=kc.cpu(), vc=vc.cpu()), dict(t=t[0]),
            dict(ks=ks[:, :0], vs=vs[:, :0]), dict(n=n.long()),
            dict(ks=ks.repeat(1, 3, 1), vs=vs.repeat(1, 3, 1)),
            dict(kc=kc[:, :, :, 1:49], vc=vc[:, :, :, 1:49])]
    bad = [lambda a=a, f=f: f(**a) for a in both for f in (attend, append)]
    bad += [lambda: attend(q=q.float()), lambda: attend(q=q[:, :3]), lambda: attend(window=0),
            lambda: attend(sinks=-1), lambda: append(k=k.half()), lambda: append(v=k[:0]),
            lambda: append(cu=cu[:1]), lambda: append(lens_out=n), lambda: append(k=k.float(), v=k),
            lambda: append(kc=kc[:1].expand(kc.shape), vc=vc[:1].expand(vc.shape)),
            lambda: append(ks=ks[:1].expand(ks.shape), vs=vs[:1].expand(vs.shape))]
    for i, f in enumerate(bad):
        with pytest.raises((TypeError, ValueError, RuntimeError)):
            f()
            print("taken:", i)
    x = k.clone().requires_grad_()
    for f in (lambda: append(k=x), lambda: append(v=x),
              lambda: attend(q=q.clone().requires_grad_())):
        with pytest.raises(RuntimeError, match="grad"):
            f()
    torch.cuda.synchronize()
