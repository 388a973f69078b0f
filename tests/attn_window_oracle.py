"""Plain 64-bit implementations of window attention and of the paged cache of 8 bits
on the host, written from their definitions, with bounds on what rounding may do to
a device result.

`head` is attn_oracle's with the pairs that are seen given, and its bounds: each
weight off by delta, rounded to 16 bits by u, sums of n terms in float32 off by
n 2^-24.

Over a cache of 8 bits (`head_scaled`) keys and values are exact: code 2^e. A weight
is 2^(y - m') with y = x + e: x, y and m' are float32, each off by half a unit in the
last place of at most |x| log2(e) + 127, four such steps to the result: delta grows by
4 (|x| 1.45 + 127 + 127) 2^-24 ln 2. In float16 a weight below 2^-14 of its type, with
2^6 for the largest, is off by 2^-25, so by 2^-31 of the largest weight times 2^e, and
meets a code; in bfloat16 the smallest weight is 2^-126 of 2^-16.
"""
import numpy as np

from attn_oracle import EPS, FLUSH, TINY, UNIT, _safe_exp


def visible(n, m, window, sinks):
    """Which of m keys each of n queries sees: the last query stands at the last key."""
    p = np.arange(n)[:, None] + (m - n)
    j = np.arange(m)[None, :]
    return (j <= p) & ((j > p - window) | (j < sinks))


def head(q, k, v, scale, seen, dtype, dout=None, out16=None):
    """One head of one sequence, `seen` [queries, keys]: {name: (value, bound)}."""
    n, m, d = q.shape[0], k.shape[0], q.shape[1]
    u, tiny = UNIT[dtype], TINY[dtype]
    x = np.full((n, m), -np.inf)
    full = (q @ k.T) * scale
    x[seen] = full[seen]
    top = x.max(1, initial=-np.inf)[:, None]
    e = np.where(seen, _safe_exp(x, top), 0.0)
    total = e.sum(1, keepdims=True)
    p = np.divide(e, total, out=np.zeros_like(e), where=total > 0)
    with np.errstate(divide="ignore"):
        lse = (np.log(total) + top)[:, 0]
    size = (np.abs(q) @ np.abs(k).T) * abs(scale)
    delta = np.where(seen, (d + 8) * EPS * size, 0.0).max(1, initial=0.0)[:, None] + 2.0 ** -20
    wide = u + 2 * delta + (m + n) * EPS
    out = p @ v
    got = {"out": (out, u * np.abs(out) + wide * (p @ np.abs(v)) +
                   (tiny + FLUSH) * (1 + seen @ np.abs(v))),
           "lse": (lse, (delta[:, 0] + 2.0 ** -20) + 2.0 ** -22 *
                   np.abs(np.where(np.isinf(lse), 0, lse)))}
    if dout is None:
        return got
    o = out if out16 is None else out16
    dp = dout @ v.T
    D = (p * dp).sum(1, keepdims=True)
    ds = scale * p * (dp - D)
    eD = np.abs((dout * (o - out)).sum(1, keepdims=True)) + \
        (d + 8) * EPS * (np.abs(dout) * np.abs(o)).sum(1, keepdims=True) + 2 * delta * np.abs(D)
    eds = (u + 2 * delta) * np.abs(ds) + abs(scale) * p * (
        2 * delta * (np.abs(dp) + np.abs(D)) + eD + (d + 8) * EPS * (np.abs(dout) @ np.abs(v).T))
    eds = eds + (m + n) * EPS * np.abs(ds)
    eds = eds + np.where(seen, FLUSH * (1 + abs(scale) * (np.abs(dp) + np.abs(D))), 0.0)
    # float16: steps of the scaled ds below its normal range, 2^-24 of the
    # largest (|ds| <= 2 scale |dout| |v|)
    if tiny and n and m:
        eds = eds + np.where(seen, 2.0 ** -36 * abs(scale) * np.linalg.norm(dout, axis=1).max() *
                             np.linalg.norm(v, axis=1).max(), 0.0)
    got["dq"] = (ds @ k, eds @ np.abs(k))
    got["dk"] = (ds.T @ q, eds.T @ np.abs(q))
    got["dv"] = (p.T @ dout, (wide * p).T @ np.abs(dout) +
                 (tiny + FLUSH) * (seen.T @ np.abs(dout)))
    return got


def packed(q, k, v, cu_q, cu_k, scale, window, sinks, dtype, dout=None, out16=None):
    """Packed sequences, grouped heads: {name: (value, bound)} in the tensors'
    layouts ([tokens, heads, head_dim]; lse [heads, tokens])."""
    T, H, d = q.shape
    K, G, _ = k.shape
    group = H // G
    got = {"out": (np.zeros((T, H, d)), np.zeros((T, H, d))),
           "lse": (np.full((H, T), -np.inf), np.zeros((H, T)))}
    if dout is not None:
        got["dq"] = (np.zeros((T, H, d)), np.zeros((T, H, d)))
        for name in ("dk", "dv"):
            got[name] = (np.zeros((K, G, d)), np.zeros((K, G, d)))
    for b in range(len(cu_q) - 1):
        i, j = slice(cu_q[b], cu_q[b + 1]), slice(cu_k[b], cu_k[b + 1])
        seen = visible(cu_q[b + 1] - cu_q[b], cu_k[b + 1] - cu_k[b], window, sinks)
        for h in range(H):
            g = h // group
            one = head(q[i, h], k[j, g], v[j, g], scale, seen, dtype,
                       None if dout is None else dout[i, h],
                       None if out16 is None else out16[i, h])
            for w in (0, 1):
                got["out"][w][i, h] = one["out"][w]
                got["lse"][w][h, i] = one["lse"][w]
                if dout is not None:
                    got["dq"][w][i, h] = one["dq"][w]
                    got["dk"][w][j, g] += one["dk"][w]
                    got["dv"][w][j, g] += one["dv"][w]
    for name in ("dq", "dk", "dv"):  # the result's own rounding
        if name in got:
            value, bound = got[name]
            bound += UNIT[dtype] * (np.abs(value) + bound) + TINY[dtype] + FLUSH
    return got


# --------------------------------------------------------------------------- #
# e4m3 codes and the cache that holds them                                    #
# --------------------------------------------------------------------------- #


def _code_values():
    """The value of each of the 256 codes: a sign, 4 bits of exponent, 3 of mantissa."""
    v = np.zeros(256)
    for c in range(256):
        e, m = c >> 3 & 15, c & 7
        x = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        if c & 127 == 127:
            x = np.nan
        v[c] = -x if c & 128 else x
    return v


CODES = _code_values()
_POSITIVE = CODES[:127]  # 0 to 448, in order


def code_of(x):
    """The code of the nearest value, ties to the even mantissa; NaN for what is not
    finite. |x| is at most 448."""
    x = np.asarray(x, np.float64)
    a = np.where(np.isfinite(x), np.abs(x), 0.0)
    hi = np.clip(np.searchsorted(_POSITIVE, a), 0, 126)
    lo = np.clip(hi - 1, 0, 126)
    up, down = _POSITIVE[hi] - a, a - _POSITIVE[lo]
    pick = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    pick = np.where(_POSITIVE[hi] == a, hi, pick)
    pick = np.where(np.isfinite(x), pick, 127)
    return (pick | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def exponent_of(values):
    """The least e of [-127, 127] with every finite |value| <= 448 * 2^e."""
    a = np.abs(np.asarray(values, np.float64).reshape(-1))
    a = a[np.isfinite(a)]
    top = a.max(initial=0.0)
    e = -127
    while top > 448 * 2.0 ** e:
        e += 1
    return e


def append_scaled(codes, scales, new, cu, table, lens):
    """`codes` [pages, page, heads, dim] and `scales` [pages, blocks, heads] with the new
    rows [tokens, heads, dim] in them (copies), and how many tokens had no place."""
    codes, scales = codes.copy(), scales.copy()
    pages, page, heads, _ = codes.shape
    block, bad = page // scales.shape[1], 0
    for b in range(len(lens)):
        n = int(cu[b + 1] - cu[b])
        places = {}
        for t in range(n):
            pos = int(lens[b]) + t
            x = int(table[b, pos // page]) if 0 <= pos < table.shape[1] * page else -1
            if 0 <= x < pages:
                places.setdefault((x, pos % page // block), []).append((pos % page, cu[b] + t))
            else:
                bad += 1
        for (x, at), tokens in places.items():
            first = tokens[0][0]
            kept = range(at * block, first)
            for h in range(heads):
                e = exponent_of([new[r, h] for _, r in tokens]) + 127
                if len(kept):
                    had = int(scales[x, at, h])
                    e = max(e, had)
                    old = codes[x, kept.start:kept.stop, h]
                    codes[x, kept.start:kept.stop, h] = code_of(CODES[old] * 2.0 ** (had - e))
                scales[x, at, h] = e
                for slot, r in tokens:
                    codes[x, slot, h] = code_of(new[r, h] * 2.0 ** (127 - e))
    return codes, scales, bad


def values_of(codes, scales):
    """What [tokens, dim] codes with [tokens] exponents' bytes stand for."""
    with np.errstate(invalid="ignore"):
        by = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
        return CODES[codes] * by[:, None]


def head_scaled(q, kc, ks, vc, vs, scale, seen, dtype):
    """One query [dim] over the tokens that it sees, codes and exponents' bytes:
    (out, bound), (lse, bound)."""
    d, u, tiny = q.shape[0], UNIT[dtype], TINY[dtype]
    kc, ks, vc, vs = kc[seen], ks[seen], vc[seen], vs[seen]
    k, v, n = values_of(kc, ks), values_of(vc, vs), kc.shape[0]
    if n == 0:
        return (np.zeros(d), np.zeros(d)), (np.array(-np.inf), np.array(0.0))
    x = k @ q * scale
    top = x.max()
    e = np.exp(x - top)
    p = e / e.sum()
    lse = np.log(e.sum()) + top
    size = (np.abs(k) @ np.abs(q)) * abs(scale)
    delta = (d + 8) * EPS * size.max() + 2.0 ** -20
    more = delta + 4 * EPS * 0.7 * (1.45 * np.abs(x).max() + 254)
    out = p @ v
    largest = (p * 2.0 ** (vs.astype(np.float64) - 127)).max()
    least = 2.0 ** -31 if tiny else 2.0 ** -110
    bound = u * np.abs(out) + (u + 2 * more + n * EPS) * (p @ np.abs(v)) + \
        least * largest * np.abs(CODES[vc]).sum(0) + tiny + FLUSH
    return (out, bound), (np.array(lse), np.array(delta + 2.0 ** -20 + 2.0 ** -22 * abs(lse)))
