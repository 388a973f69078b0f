"""Plain 64-bit implementations of the attention operators on the host, written
from their definitions, with bounds on what rounding may do to a device result.

Bounds. u is half a unit in the last place of the 16-bit type, relative to the
value: 2^-8 for bfloat16 (8 bits with the leading one), 2^-11 for float16 (11);
tiny its smallest step, for float16's small values. FLUSH: float32 and bfloat16
values below 2^-126 may become zero (weights, ds, results).
Scores are float32 sums of exact products, off by at most
(head_dim + 8) 2^-24 sum|q k| scale, and their exponentials by 2^-20 more
(relative): together delta on each weight and on their sum. Rounding the weights
to 16 bits adds u, float32 sums of n terms n 2^-24. So

  out  <= u |out| + (u + 2 delta + n 2^-24) sum p|v|
  lse  <= delta + 2^-22 |lse| + 2^-20
  dv   <= u |dv| + (u + 2 delta + n 2^-24) sum p|dout|
  D    <= u sum|dout out| + head_dim 2^-24 sum|dout out|: out is 16 bits
  ds   <= (u + 2 delta) |ds| + scale p (2 delta (|dp| + |D|) + err D
          + head_dim 2^-24 sum|dout v|)
  dq, dk: their own rounding and the sums of err ds |k|, |q|.
"""
import numpy as np

UNIT = {"bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}
TINY = {"bfloat16": 0.0, "float16": 2.0 ** -25}
EPS = 2.0 ** -24
FLUSH = 2.0 ** -126


def _safe_exp(x, top):
    return np.exp(x - np.where(np.isneginf(top), 0.0, top))


def head(q, k, v, scale, causal, dtype, dout=None, out16=None):
    """One head of one sequence: {name: (value, bound)}. out16: the 16-bit output
    that the gradient is given (its error is part of the bound)."""
    n, m, d = q.shape[0], k.shape[0], q.shape[1]
    u, tiny = UNIT[dtype], TINY[dtype]
    seen = np.ones((n, m), bool)
    if causal:
        seen = np.arange(m)[None, :] <= np.arange(n)[:, None] + (m - n)
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
                   (tiny + FLUSH) * (1 + np.abs(v).sum(0)[None, :])),
           "lse": (lse, (delta[:, 0] + 2.0 ** -20) + 2.0 ** -22 *
                   np.abs(np.where(np.isinf(lse), 0, lse)))}
    if dout is None:
        return got
    o = out if out16 is None else out16
    dp = dout @ v.T
    D = (p * dp).sum(1, keepdims=True)
    ds = scale * p * (dp - D)
    eD = np.abs((dout * (o - out)).sum(1, keepdims=True)) + \
        (d + 8) * EPS * (np.abs(dout) * np.abs(o)).sum(1, keepdims=True) + \
        2 * delta * np.abs(D)
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
                 (tiny + FLUSH) * np.abs(dout).sum(0)[None, :])
    return got


def packed(q, k, v, cu_q, cu_k, scale, causal, dtype, dout=None, out16=None):
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
        for h in range(H):
            g = h // group
            one = head(q[i, h], k[j, g], v[j, g], scale, causal, dtype,
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


def fork(page, pages, table, lens, parent, room, held=None):
    """The next page table by its definition: (table, lens, refs, copies), copies
    a list of (from, to)."""
    rows, width = table.shape[0], table.shape[1]
    used = np.zeros(pages, np.int64)
    out = np.full((len(parent), width), -1, np.int64)
    new_lens = np.zeros(len(parent), np.int64)
    wants = []
    taken = set()
    for i, p in enumerate(parent):
        p = p if 0 <= p < rows else -1
        n = min(max(int(lens[p]), 0), width * page) if p >= 0 else 0
        keep = n // page
        copy = False
        if n % page:
            if p in taken:
                copy = True
            else:
                keep += 1
            taken.add(p)
        for s in range(keep):
            x = int(table[p, s])
            if 0 <= x < pages:
                out[i, s] = x
                used[x] += 1
        new_lens[i] = n
        top = min(max(n, int(room[i]) if room is not None else n), width * page)
        for s in range(keep, -(-top // page)):
            wants.append((i, s, p if copy and s == n // page else None))
    free = [x for x in range(pages) if not used[x] and not (held is not None and held[x] > 0)]
    copies = []
    for (i, s, p), x in zip(wants, free):
        out[i, s] = x
        used[x] += 1
        if p is not None:
            copies.append((int(table[p, s]), x))
    for i, s, p in wants[len(free):]:
        if p is not None:
            new_lens[i] = s * page
    refs = used + (held if held is not None else 0)
    return out, new_lens, refs, copies, len(wants) > len(free)


def compact(pages, table, held=None):
    """(table, moved, live, moves)."""
    used = np.zeros(pages, bool)
    for x in table.reshape(-1):
        if 0 <= x < pages:
            used[x] = True
    if held is not None:
        used |= held > 0
    m = int(used.sum())
    holes = [x for x in range(m) if not used[x]]
    highs = [x for x in range(m, pages) if used[x]]
    moved = np.where(used, np.arange(pages), -1)
    for x, y in zip(highs, holes):
        moved[x] = y
    out = np.array([moved[x] if 0 <= x < pages else -1 for x in table.reshape(-1)],
                   np.int64).reshape(table.shape)
    return out, moved, m, list(zip(highs, holes))
