"""Timing cases of the attention workload: the operators that a profiled
language model spends its kernel time in, from the prompt to the cache.

Each case is one pass of one of them, over seeded inputs made on the GPU:

prompt    attention over whole prompts, sequences of different lengths packed
          one after another, grouped heads
train     the same and its gradient: a training step's share
step      one new token a sequence: its keys and values go into the paged
          cache, its queries read the cache
append    keys and values of whole prompts written into the paged cache
turn      a scheduler's turn between steps: sequences dropped, kept, forked and
          given room for more, then the pages in use moved together

A case is a dict of plain values:

seqs, longest   sequences (rows of the page table) and the longest's tokens
pick            0: every sequence is the longest; else a number that picks
                their lengths, from one token to the longest, evenly over the
                logarithm
heads, kv_heads, dim   query heads, key and value heads, values a head
before          prompt, train: keys that each sequence had before the prompt
causal          prompt, train: later keys are masked
dtype           bfloat16 | float16
page            tokens a page
planes          turn: pools that share one page table (keys and values a layer)
pages           turn: pages in the pool
"""
import math
import random

import torch

own = False

DEV = "cuda:0"
TYPES = {"bfloat16": torch.bfloat16, "float16": torch.float16}


def listed():
    return [
        # GPT-2's shape: four short prompts, twelve heads, where a pass is
        # mostly the cost of a launch
        dict(name="prompt-4x128", op="prompt", seqs=4, longest=128, pick=0, heads=12,
             kv_heads=12, dim=64, before=0, causal=True, dtype="bfloat16"),
        # prompts as a server packs them: a few long ones, most of them short,
        # odd lengths, four query heads to a key head
        dict(name="prompt-packed-24", op="prompt", seqs=24, longest=4099, pick=7, heads=32,
             kv_heads=8, dim=128, before=0, causal=True, dtype="bfloat16"),
        # one long document
        dict(name="prompt-long-16k", op="prompt", seqs=1, longest=16384, pick=0, heads=16,
             kv_heads=4, dim=128, before=0, causal=True, dtype="float16"),
        # the SDPA workload's shape, no mask, with its gradient
        dict(name="train-8x512", op="train", seqs=8, longest=512, pick=0, heads=8, kv_heads=8,
             dim=64, before=0, causal=False, dtype="bfloat16"),
        # a training batch of packed documents, grouped heads
        dict(name="train-packed-12", op="train", seqs=12, longest=4001, pick=5, heads=16,
             kv_heads=4, dim=128, before=0, causal=True, dtype="bfloat16"),
        # a few short answers under way
        dict(name="step-4x150", op="step", seqs=4, longest=150, pick=0, heads=12, kv_heads=12,
             dim=64, page=16, dtype="bfloat16"),
        # a full serving batch, every sequence somewhere else in its answer
        dict(name="step-96-mixed", op="step", seqs=96, longest=9001, pick=3, heads=32,
             kv_heads=8, dim=128, page=16, dtype="bfloat16"),
        # two sequences with long caches: few rows, one long axis
        dict(name="step-2x131k", op="step", seqs=2, longest=131_000, pick=0, heads=32,
             kv_heads=8, dim=128, page=64, dtype="float16"),
        # a short prompt enters the cache
        dict(name="append-77", op="append", seqs=1, longest=77, pick=0, heads=12, kv_heads=12,
             dim=64, page=16, dtype="bfloat16"),
        # a prefill's keys and values enter the cache
        dict(name="append-packed-40", op="append", seqs=40, longest=16000, pick=9, heads=32,
             kv_heads=8, dim=128, page=16, dtype="bfloat16"),
        # a small scheduler's turn: twelve layers, eight sequences
        dict(name="turn-8", op="turn", seqs=8, longest=300, pick=2, heads=12, kv_heads=12,
             dim=64, page=16, planes=24, pages=256, dtype="bfloat16"),
        # a large one: many sequences sharing a pool
        dict(name="turn-160", op="turn", seqs=160, longest=4096, pick=4, heads=32, kv_heads=8,
             dim=128, page=16, planes=8, pages=8192, dtype="bfloat16"),
    ]


def _spread(rng, low, high):
    """A whole number of [low, high], evenly over the logarithm."""
    return min(high, int(math.exp(rng.uniform(math.log(low), math.log(high + 1)))))


def draw(rng):
    op = rng.choice(("prompt", "train", "step", "append", "turn"))
    dim = rng.choice((64, 128))
    kv = rng.choice((1, 2, 4, 8, 12))
    heads = kv * rng.choice((1, 2, 3, 4, 8))
    heads = kv if heads > 32 else heads
    case = dict(op=op, pick=rng.randrange(1, 10_000), heads=heads, kv_heads=kv, dim=dim,
                dtype=rng.choice(("bfloat16", "float16")))
    if op in ("prompt", "train"):
        longest = _spread(rng, 60, 9000 if op == "prompt" else 4000)
        # the plain form holds sequences x heads x longest^2 scores
        most = int(16 * 16384 ** 2 / (longest ** 2 * heads))
        case.update(longest=longest, seqs=_spread(rng, 1, max(1, min(32, most))),
                    before=rng.choice((0, 0, rng.randrange(1, longest))) // 2,
                    causal=rng.random() < 0.75)
    elif op == "step":
        seqs = _spread(rng, 1, 128)
        case.update(seqs=seqs, longest=_spread(rng, 40, 262_000 // seqs + 2000),
                    page=rng.choice((16, 32, 64)))
    elif op == "append":
        seqs = _spread(rng, 1, 64)
        case.update(seqs=seqs, longest=_spread(rng, 2, 60_000 // seqs + 1000),
                    page=rng.choice((16, 32, 64)))
    else:
        page = rng.choice((16, 32))
        seqs = _spread(rng, 2, 160)
        longest = _spread(rng, page, 4096)
        case.update(seqs=seqs, longest=longest, page=page, planes=2 * rng.choice((1, 2, 4)))
        # room for the rows held, the rows forked and what they are given
        want = sum(-(-n // page) for n in _lengths(case))
        case["pages"] = int(want * rng.uniform(2.1, 3.0)) + 8 * seqs
    return case


def _lengths(case):
    """Tokens of each sequence: the first is the longest."""
    n, longest = case["seqs"], case["longest"]
    if not case["pick"]:
        return [longest] * n
    rng = random.Random(case["pick"])
    return [longest] + [_spread(rng, 1, longest) for _ in range(n - 1)]


def _starts(lengths):
    at = [0]
    for n in lengths:
        at.append(at[-1] + n)
    return at


def _visible(case):
    """Pairs of a query and a key that it sees, over one head."""
    b, pairs = case["before"], 0
    for n in _lengths(case):
        pairs += n * b + n * (n + 1) // 2 if case["causal"] else n * (n + b)
    return pairs


def _turn_rows(case):
    """What the scheduler decides: the row that each row of the next table
    continues (-1: a new one), and the tokens it wants room for. A fifth of the
    rows end, a quarter are forked once or twice, the rest go on."""
    rng = random.Random(case["pick"] + 1)
    parent = []
    for row in range(case["seqs"]):
        parent += [row] * rng.choice((0, 1, 1, 1, 1, 1, 1, 2, 2, 3))
    parent = parent[:case["seqs"]]
    parent += [-1] * (case["seqs"] - len(parent))
    lengths = _lengths(case)
    room = [(lengths[p] if p >= 0 else 0) + rng.randrange(1, 2 * case["page"]) for p in parent]
    return parent, room


def work(case):
    h, g, d = case["heads"], case["kv_heads"], case["dim"]
    tokens = sum(_lengths(case))
    if case["op"] in ("prompt", "train"):
        keys = tokens + case["before"] * case["seqs"]
        pairs = _visible(case) * h
        # q, k, v read; out and the row statistic written
        moved = 2 * d * (2 * tokens * h + 2 * keys * g) + 4 * tokens * h
        if case["op"] == "prompt":
            return {"bytes": moved, "flops": 4 * d * pairs}
        # the gradient reads these again with out's gradient, and writes three
        moved += 2 * d * (3 * tokens * h + 2 * keys * g) + 4 * tokens * h
        moved += 2 * d * (tokens * h + 2 * keys * g)
        return {"bytes": moved, "flops": 14 * d * pairs}
    if case["op"] == "step":
        return {"bytes": 2 * d * (2 * g * tokens + 2 * h * case["seqs"]) + 4 * tokens // case["page"],
                "flops": 4 * d * h * tokens}
    if case["op"] == "append":
        return {"bytes": 2 * 2 * d * 2 * g * tokens, "flops": 0}
    # turn: the copied last pages of the forks; pages in use above the count of
    # pages in use, moved below it (they lie anywhere: a share of them does)
    parent, room = _turn_rows(case)
    page, lengths = case["page"], _lengths(case)
    copies = sum(p >= 0 and p in parent[:i] and lengths[p] % page > 0
                 for i, p in enumerate(parent))
    kept = sum(-(-lengths[p] // page) for p in set(parent) if p >= 0)
    more = copies + sum(-(-r // page) - (-(-lengths[p] // page) if p >= 0 else 0)
                        for p, r in zip(parent, room))
    live = kept + more
    moves = int(kept * max(0.0, 1 - live / case["pages"]))
    plane = page * g * d * 2
    tables = 8 * case["seqs"] * _width(case) + 8 * case["pages"]
    return {"bytes": 2 * case["planes"] * plane * (copies + moves) + tables, "flops": 0}


def _width(case):
    """Columns of the page table: the longest sequence and room beside it."""
    return -(-case["longest"] // case["page"]) + 3


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _page_table(case, lengths, gen, pages=None):
    """Pages of each sequence, anywhere in the pool, -1 past the last."""
    page, width = case["page"], _width(case)
    counts = [-(-n // page) for n in lengths]
    pages = pages or sum(counts) + 5
    order = torch.randperm(pages, generator=gen, device=DEV)[:sum(counts)].to(torch.int32)
    slot = torch.arange(width, device=DEV)[None, :]
    count = _ints(counts)[:, None]
    first = (torch.cumsum(count, 0) - count).long()
    at = (first + slot).clamp(max=max(0, sum(counts) - 1))
    table = torch.where(slot < count, order[at], torch.full_like(at, -1, dtype=torch.int32))
    return table.to(torch.int32).contiguous(), pages


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(1_000_003 * seed + 17)
    dtype = TYPES[case["dtype"]]
    h, g, d = case["heads"], case["kv_heads"], case["dim"]
    lengths = _lengths(case)
    tokens = sum(lengths)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=DEV, dtype=torch.float32)

    s = dict(case=dict(case), scale=1.0 / math.sqrt(d), ws=None)
    if case["op"] in ("prompt", "train"):
        # heads of different sharpness, as trained ones are; queries, keys and
        # values side by side in a row, as the projection leaves them
        sharp = torch.linspace(0.5, 2.5, h, device=DEV)[None, :, None]
        rows = torch.empty(tokens, h + 2 * g, d, dtype=dtype, device=DEV)
        rows[:, :h] = normal(tokens, h, d) * sharp
        rows[:, h:] = normal(tokens, 2 * g, d)
        s["q"] = rows[:, :h]
        keys = [n + case["before"] for n in lengths]
        if case["before"]:
            kv = normal(sum(keys), 2 * g, d).to(dtype)
            s["k"], s["v"] = kv[:, :g], kv[:, g:]
        else:
            s["k"], s["v"] = rows[:, h:h + g], rows[:, h + g:]
        s["cu_q"], s["cu_k"] = _ints(_starts(lengths)), _ints(_starts(keys))
        s["most_q"], s["most_k"] = max(lengths), max(keys)
        s["out"] = torch.empty(tokens, h, d, dtype=dtype, device=DEV)
        s["lse"] = torch.empty(h, tokens, dtype=torch.float32, device=DEV)
        if case["op"] == "train":
            s["dout"] = (0.1 * normal(tokens, h, d)).to(dtype)
            s["dq"] = torch.empty(tokens, h, d, dtype=dtype, device=DEV)
            s["dk"] = torch.empty(sum(keys), g, d, dtype=dtype, device=DEV)
            s["dv"] = torch.empty(sum(keys), g, d, dtype=dtype, device=DEV)
        return s
    if case["op"] == "turn":
        s["table"], _ = _page_table(case, lengths, gen, case["pages"])
        s["lens"] = _ints(lengths)
        parent, room = _turn_rows(case)
        s["parent"], s["room"] = _ints(parent), _ints(room)
        s["pool"] = torch.randint(-2 ** 31, 2 ** 31 - 1, (case["planes"], case["pages"],
                                                          case["page"] * g * d // 2),
                                  generator=gen, device=DEV, dtype=torch.int32).view(dtype)
        return s
    # one cache of keys and values, as a layer of a server holds it
    s["table"], pages = _page_table(case, lengths, gen)
    cache = torch.empty(2, pages, case["page"], g, d, dtype=dtype, device=DEV)
    cache[0] = normal(pages, case["page"], g, d)
    cache[1] = normal(pages, case["page"], g, d)
    s["cache"] = cache
    if case["op"] == "step":
        rows = normal(case["seqs"], h + 2 * g, d)
        rows[:, :h] *= torch.linspace(0.5, 2.5, h, device=DEV)[None, :, None]
        # a sequence that is only one token long has nothing in the cache yet
        s["lens"] = _ints([n - 1 for n in lengths])
        s["cu"] = _ints(list(range(case["seqs"] + 1)))
        s["out"] = torch.empty(case["seqs"], h, d, dtype=dtype, device=DEV)
        s["lse"] = torch.empty(h, case["seqs"], dtype=torch.float32, device=DEV)
    else:
        rows = normal(tokens, h + 2 * g, d)
        s["lens"] = torch.zeros(case["seqs"], dtype=torch.int32, device=DEV)
        s["cu"] = _ints(_starts(lengths))
    rows = rows.to(dtype)
    s["q"], s["k"], s["v"] = rows[:, :h], rows[:, h:h + g], rows[:, h + g:]
    s["after"] = torch.empty(case["seqs"], dtype=torch.int32, device=DEV)
    return s


def run(s):
    op = s["case"]["op"]
    if own:
        return _OWN[op](s)
    return _PLAIN[op](s)


# --------------------------------------------------------------------------- #
# the framework's calls                                                       #
# --------------------------------------------------------------------------- #


def _workspace(s):
    from paper_2609_11938_amd import opattr

    if s["ws"] is None:
        s["ws"] = opattr.Workspace(DEV)
    return s["ws"]


def _own_prompt(s):
    from paper_2609_11938_amd import attn

    return attn.opattr_attn_prompt(s["q"], s["k"], s["v"], s["cu_q"], s["cu_k"],
                                   causal=s["case"]["causal"], scale=s["scale"], out=s["out"],
                                   lse=s["lse"])


def _own_train(s):
    from paper_2609_11938_amd import attn

    out, lse = _own_prompt(s)
    dq, dk, dv = attn.opattr_attn_prompt_grad(
        s["dout"], s["q"], s["k"], s["v"], out, lse, s["cu_q"], s["cu_k"],
        causal=s["case"]["causal"], scale=s["scale"], dq=s["dq"], dk=s["dk"], dv=s["dv"],
        ws=_workspace(s))
    return out, lse, dq, dk, dv


def _own_append(s):
    from paper_2609_11938_amd import attn

    attn.opattr_kv_append(s["k"], s["v"], s["cu"], s["cache"][0], s["cache"][1], s["table"],
                          s["lens"], lens_out=s["after"])
    return s["cache"].view(torch.int16), s["after"]


def _own_step(s):
    from paper_2609_11938_amd import attn

    cache, after = _own_append(s)
    out, lse = attn.opattr_attn_paged(s["q"], s["cache"][0], s["cache"][1], s["table"], after,
                                      scale=s["scale"], out=s["out"], lse=s["lse"],
                                      ws=_workspace(s))
    return out, lse, cache, after


def _own_turn(s):
    from paper_2609_11938_amd import attn

    page, ws = s["case"]["page"], _workspace(s)
    f = attn.opattr_pages_fork(s["pool"], page, s["table"], s["lens"], s["parent"], s["room"],
                               ws=ws)
    c = attn.opattr_pages_compact(s["pool"], f["table"], ws=ws)
    return (c["table"], f["lens"], f["refs"], c["moved"], c["live"], s["pool"].view(torch.int16))


_OWN = dict(prompt=_own_prompt, train=_own_train, step=_own_step, append=_own_append,
            turn=_own_turn)

# --------------------------------------------------------------------------- #
# the plain forms                                                             #
# --------------------------------------------------------------------------- #


def _padded(rows, cu, most):
    """[sequences, heads, most, dim] in 32 bits, the place of each row in it,
    and which of its rows are there."""
    at = cu[:-1, None].long() + torch.arange(most, device=DEV)[None, :]
    there = at < cu[1:, None]
    at = at.clamp(max=max(0, rows.shape[0] - 1))
    full = rows.float()[at] * there[:, :, None, None]
    return full.transpose(1, 2).contiguous(), there


def _packed(full, there, dtype):
    return full.transpose(1, 2)[there].to(dtype)


def _scores(s):
    """Queries, keys and values as padded rows (each key head repeated for its
    queries), the masked scores, and which rows are there."""
    case = s["case"]
    group = case["heads"] // case["kv_heads"]
    q, there_q = _padded(s["q"], s["cu_q"], s["most_q"])
    k, there_k = _padded(s["k"], s["cu_k"], s["most_k"])
    v, _ = _padded(s["v"], s["cu_k"], s["most_k"])
    k, v = k.repeat_interleave(group, 1), v.repeat_interleave(group, 1)
    seen = there_k[:, None, None, :]
    if case["causal"]:
        lead = (s["cu_k"][1:] - s["cu_k"][:-1]) - (s["cu_q"][1:] - s["cu_q"][:-1])
        i = torch.arange(s["most_q"], device=DEV)[None, :, None] + lead[:, None, None]
        j = torch.arange(s["most_k"], device=DEV)[None, None, :]
        seen = seen & (j <= i)[:, None]
    x = torch.matmul(q, k.transpose(2, 3)).mul_(s["scale"])
    x.masked_fill_(~seen, -math.inf)
    return q, k, v, x, there_q, there_k


def _softmax(x):
    """The rows' weights (in place of the scores) and the logarithm of their
    sum; rows that see nothing have weights 0 and -inf."""
    top = x.amax(-1, keepdim=True)
    x.sub_(torch.where(top == -math.inf, torch.zeros_like(top), top)).exp_()
    total = x.sum(-1, keepdim=True)
    x.div_(torch.where(total == 0, torch.ones_like(total), total))
    return x, (top + total.log()).squeeze(-1)


def _plain_prompt(s):
    dtype = TYPES[s["case"]["dtype"]]
    _, _, v, x, there, _ = _scores(s)
    p, lse = _softmax(x)
    out = torch.matmul(p, v)
    return _packed(out, there, dtype), lse.transpose(1, 2)[there].t().contiguous()


def _plain_train(s):
    case, dtype = s["case"], TYPES[s["case"]["dtype"]]
    group = case["heads"] // case["kv_heads"]
    q, k, v, x, there, there_k = _scores(s)
    p, lse = _softmax(x)
    out = torch.matmul(p, v)
    do, _ = _padded(s["dout"], s["cu_q"], s["most_q"])

    def grouped(t):
        b, _, n, d = t.shape
        return t.view(b, case["kv_heads"], group, n, d).sum(2)

    dv = grouped(torch.matmul(p.transpose(2, 3), do))
    dx = torch.matmul(do, v.transpose(2, 3)).sub_((do * out).sum(-1, keepdim=True)).mul_(p)
    dx.mul_(s["scale"])
    dq = torch.matmul(dx, k)
    dk = grouped(torch.matmul(dx.transpose(2, 3), q))
    return (_packed(out, there, dtype), lse.transpose(1, 2)[there].t().contiguous(),
            _packed(dq, there, dtype), _packed(dk, there_k, dtype), _packed(dv, there_k, dtype))


def _plain_append(s):
    page = s["case"]["page"]
    cu, tokens = s["cu"].long(), s["k"].shape[0]
    t = torch.arange(tokens, device=DEV)
    row = torch.searchsorted(cu, t, right=True) - 1
    at = t - cu[row] + s["lens"].long()[row]
    to = s["table"].long()[row, at // page]
    s["cache"][0][to, at % page] = s["k"]
    s["cache"][1][to, at % page] = s["v"]
    after = s["lens"] + (s["cu"][1:] - s["cu"][:-1])
    return s["cache"].view(torch.int16), after


def _plain_step(s):
    case, dtype = s["case"], TYPES[s["case"]["dtype"]]
    cache, after = _plain_append(s)
    b, g, d = case["seqs"], case["kv_heads"], case["dim"]
    table = s["table"].long().clamp(min=0)
    k = s["cache"][0][table].float().view(b, -1, g, d).transpose(1, 2)
    v = s["cache"][1][table].float().view(b, -1, g, d).transpose(1, 2)
    q = s["q"].float().view(b, g, case["heads"] // g, d)
    x = torch.matmul(q, k.transpose(2, 3)).mul_(s["scale"])
    seen = torch.arange(x.shape[-1], device=DEV)[None, :] < after[:, None]
    x.masked_fill_(~seen[:, None, None, :], -math.inf)
    p, lse = _softmax(x)
    out = torch.matmul(p, v).view(b, case["heads"], d).to(dtype)
    return out, lse.view(b, case["heads"]).t().contiguous(), cache, after


def _plain_turn(s):
    case = s["case"]
    page, width, pages = case["page"], s["table"].shape[1], case["pages"]
    # fork: a child takes its parent's full pages; the part-filled last page
    # stays with the first child and is copied for the others
    parent = s["parent"].long()
    lens = torch.where(parent >= 0, s["lens"].long()[parent.clamp(min=0)], 0)
    full, part = lens // page, lens % page
    same = (parent[:, None] == parent[None, :]) & (parent >= 0)[:, None]
    first = ~torch.tril(same, -1).any(1)
    slot = torch.arange(width, device=DEV)[None, :]
    last = (slot == full[:, None]) & (part > 0)[:, None]
    kept = (slot < full[:, None]) | (last & first[:, None])
    want = (torch.maximum(s["room"].long(), lens) + page - 1) // page
    new = (slot < want[:, None]) & ~kept
    old = s["table"].long()[parent.clamp(min=0)]
    used = torch.bincount(old[kept], minlength=pages)
    free = torch.nonzero(used == 0).squeeze(1)
    rank = torch.cumsum(new.reshape(-1).long(), 0).view_as(new) - 1
    table = torch.where(kept, old, torch.where(new, free[rank.clamp(min=0)], -1))
    copied = last & ~first[:, None]
    s["pool"][:, table[copied]] = s["pool"][:, old[copied]]
    refs = torch.bincount(table[table >= 0], minlength=pages)
    # compact: the pages in use past their count go to the holes below it
    count = (refs > 0).sum()
    spot = torch.arange(pages, device=DEV)
    source = torch.nonzero((refs > 0) & (spot >= count)).squeeze(1)
    hole = torch.nonzero((refs == 0) & (spot < count)).squeeze(1)
    moved = torch.where(refs > 0, spot, -1)
    moved[source] = hole
    s["pool"][:, hole] = s["pool"][:, source]
    table = torch.where(table >= 0, moved[table.clamp(min=0)], -1)
    return (table.to(torch.int32), lens.to(torch.int32), refs.to(torch.int32),
            moved.to(torch.int32), count.to(torch.int32).view(1), s["pool"].view(torch.int16))


_PLAIN = dict(prompt=_plain_prompt, train=_plain_train, step=_plain_step, append=_plain_append,
              turn=_plain_turn)

# --------------------------------------------------------------------------- #
# the definition in 64 bits                                                   #
# --------------------------------------------------------------------------- #


def _exact_head(q, k, v, scale, causal, dout=None):
    """Attention of one head of one sequence, its row statistic, and the
    gradients for `dout`."""
    x = q @ k.T * scale
    if causal:
        i = torch.arange(q.shape[0], device=DEV)[:, None] + (k.shape[0] - q.shape[0])
        x = x.masked_fill(torch.arange(k.shape[0], device=DEV)[None, :] > i, -math.inf)
    lse = torch.logsumexp(x, 1)
    p = torch.exp(x - lse[:, None])
    out = p @ v
    if dout is None:
        return out, lse
    dp = dout @ v.T
    dx = p * (dp - (p * dp).sum(1, keepdim=True)) * scale
    return out, lse, dx @ k, dx.T @ q, p.T @ dout


def exact(case, seed):
    if case["op"] in ("append", "turn"):
        return None  # whole numbers: copies, tables and counts
    s = prepare(case, seed)
    group, lengths = case["heads"] // case["kv_heads"], _lengths(case)
    if case["op"] == "step":
        out = torch.empty(case["seqs"], case["heads"], case["dim"], dtype=torch.float64,
                          device=DEV)
        lse = torch.empty(case["heads"], case["seqs"], dtype=torch.float64, device=DEV)
        for b, n in enumerate(lengths):
            where = s["table"][b, :-(-n // case["page"])].long()
            k = s["cache"][0][where].double().flatten(0, 1)[:n]
            v = s["cache"][1][where].double().flatten(0, 1)[:n]
            k[n - 1], v[n - 1] = s["k"][b].double(), s["v"][b].double()
            for g in range(case["kv_heads"]):
                h = slice(g * group, (g + 1) * group)
                out[b, h], lse[h, b] = _exact_head(s["q"][b, h].double(), k[:, g], v[:, g],
                                                   s["scale"], False)
        return out, lse, None, None
    train = case["op"] == "train"
    like = dict(dtype=torch.float64, device=DEV)
    out, lse = torch.empty(s["q"].shape, **like), torch.empty(s["lse"].shape, **like)
    dq, dk, dv = (torch.zeros(t.shape, **like) for t in (s["q"], s["k"], s["v"]))
    at_q = _starts(lengths)
    at_k = _starts([n + case["before"] for n in lengths])
    for b in range(case["seqs"]):
        i, j = slice(at_q[b], at_q[b + 1]), slice(at_k[b], at_k[b + 1])
        for h in range(case["heads"]):
            g = h // group
            got = _exact_head(s["q"][i, h].double(), s["k"][j, g].double(),
                              s["v"][j, g].double(), s["scale"], case["causal"],
                              s["dout"][i, h].double() if train else None)
            out[i, h], lse[h, i] = got[:2]
            if train:
                dq[i, h] = got[2]
                dk[j, g] += got[3]
                dv[j, g] += got[4]
    return (out, lse, dq, dk, dv) if train else (out, lse)
