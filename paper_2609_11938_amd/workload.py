"""A language model's attention, served and trained with the operators of
``attn`` and profiled with the attribution join of ``opattr``: a real trace of
this GPU next to the synthetic ones of ``tracegen``.

    python -m paper_2609_11938_amd.workload profile.json [--window N] [--sinks N] [--scaled]

``serve`` takes prompts into a paged cache, generates tokens, and between them
forks, drops and compacts sequences as a scheduler does; ``train`` runs the
forward pass and its gradient over packed documents. Both take a sliding window with
sinks, and ``serve`` a cache of 8 bits. Rows of random numbers
stand for the projections' outputs. Every call is recorded by a ``Recorder``
(device time by events, with the host kept ahead; bytes as the call has to move them, computed from its
sizes and results, not counted in the memory: rows, and of a cache what is in it; an append's
exponents, and what it rounds again as they grow, are not among them) inside the operator range that
issued it; ``profile`` attributes the trace and builds the profile document.
"""
from __future__ import annotations

import argparse
import contextlib
import functools
import math
import sys

import numpy as np
import torch

from . import attn, opattr
from . import profile as profile_doc

# counters a Recorder fills (the rest are absent): time, bytes read and written
TIME, READ, WRITTEN = 0, 1, 2
ABSENT = ((1 << opattr.NUM_COUNTERS) - 1) & ~(1 << TIME | 1 << READ | 1 << WRITTEN)


# Clock cycles that the device waits before a recorded call, so that the host is done
# with the call before the device begins: about 0.2 ms, for calls that cost the host
# 4 to 20 us.
AHEAD = 500_000


class Recorder:
    """Launch records and operator ranges of calls on the current stream. ``late``
    counts the calls that the device began before the host was done with them:
    their times hold some of the host's."""

    def __init__(self):
        self.names, self.ops = [], []
        self.launches, self.ranges, self.open = [], [], []
        self.late = 0
        self.base = self._event()
        self.idle = 0.0  # ms between two events with nothing in between
        nothing = [self._timed(lambda: None)[1:] for _ in range(15)]
        torch.cuda.synchronize()
        self.idle = sorted(a.elapsed_time(b) for a, b in nothing)[7]
        self.late = 0

    @staticmethod
    def _event():
        e = torch.cuda.Event(enable_timing=True)
        e.record()
        return e

    def _timed(self, call, *args, **kw):
        torch.cuda._sleep(AHEAD)
        begin = self._event()
        result = call(*args, **kw)
        end = self._event()
        self.late += begin.query()
        return result, begin, end

    @staticmethod
    def _id(names, name):
        if name not in names:
            names.append(name)
        return names.index(name)

    @contextlib.contextmanager
    def op(self, name):
        """An operator range around what is recorded inside."""
        at = len(self.ranges)
        self.ranges.append([self._id(self.ops, name), len(self.launches), 0])
        self.open.append(at)
        yield
        self.open.pop()
        self.ranges[at][2] = len(self.launches)

    def launch(self, name, read, written, call, *args, **kw):
        """call(*args, **kw), recorded as one launch, whatever kernels it takes. Bytes
        that depend on the data are functions of the result, called by trace()."""
        result, begin, end = self._timed(call, *args, **kw)
        moved = [functools.partial(n, result) if callable(n) else n for n in (read, written)]
        self.launches.append((self._id(self.names, name), begin, end, *moved))
        return result

    def trace(self) -> dict:
        """The host trace (see opattr.to_device): one stream, every launch profiled."""
        torch.cuda.synchronize()
        T = len(self.launches)
        start = np.zeros(T, np.uint64)
        dur = np.zeros(T, np.uint32)
        counters = np.zeros((T, opattr.NUM_COUNTERS), np.float32)
        last = 0
        for i, (_, begin, end, read, written) in enumerate(self.launches):
            # events have their own resolution: a launch starts at or after the
            # end of the one before it
            s = max(last, round(self.base.elapsed_time(begin) * 1e6))
            d = max(1, round((begin.elapsed_time(end) - self.idle) * 1e6))
            start[i], dur[i], last = s, d, s + d
            counters[i, [TIME, READ, WRITTEN]] = d, *(n() if callable(n) else n
                                                       for n in (read, written))
        ranges = [(o, a, b) for o, a, b in self.ranges if b > a]
        first, final = (np.array([r[k] for r in ranges], np.int64) for k in (1, 2))
        name = np.array([n for n, *_ in self.launches], np.uint32)
        end = start + dur
        return dict(seq=np.arange(T, dtype=np.uint32), start_ns=start, dur_ns=dur,
                    stream_id=np.zeros(T, np.uint16), name_id=name, pf_name=name.copy(),
                    counters=counters, r_start=start[first], r_end=end[final - 1],
                    r_stream=np.zeros(len(ranges), np.uint16),
                    r_op=np.array([r[0] for r in ranges], np.uint32),
                    n_names=max(1, len(self.names)), n_streams=1, n_ops=max(1, len(self.ops)))


def profile(rec: Recorder, **metadata) -> dict:
    """The recorded trace attributed to its operators: the profile document."""
    tr = rec.trace()
    dt = opattr.to_device(tr)
    flags = opattr.KERNELS_STREAM_MAJOR | opattr.SEQ_DENSE | opattr.RANGES_NESTED
    out = opattr.opattr_attribute(dt, flags=flags, absent_mask=ABSENT)
    disp = opattr.opattr_aggregate_dispatch(dt, out["match"], out["range_id"], flags=flags,
                                            absent_mask=ABSENT)
    torch.cuda.synchronize()
    rid = out["range_id"].cpu().numpy()
    op = np.where(rid >= 0, tr["r_op"].astype(np.int64)[np.maximum(rid, 0)], -1)
    tier = np.where(rid >= 0, opattr.TIER_NVTX, opattr.TIER_UNATTRIBUTED)
    return profile_doc.build(tr, out["match"].cpu().numpy(), tier, op, np.zeros_like(tier),
                             disp["row"].cpu().numpy(), disp.table_host(),
                             op_names=rec.ops, kernel_names=rec.names,
                             metadata={"model_name": "attention workload",
                                       "late_launches": rec.late, **metadata},
                             absent_mask=ABSENT)


class Cache:
    """A paged cache of several layers: one pool [layers, 2, pages, page_size,
    kv_heads, head_dim], one page table, one length a sequence. scaled: of 8 bits, a
    page's exponents (one for `block` tokens of a head) behind its codes, so that turns
    take both along; `data` holds the codes and `scales` the exponents."""

    def __init__(self, layers, pages, page_size, kv_heads, head_dim, rows, width,
                 dtype=torch.bfloat16, device="cuda:0", scaled=False, block=None):
        ints = dict(dtype=torch.int32, device=device)
        self.page_size, self.layers = page_size, layers
        shape = (layers, 2, pages, page_size, kv_heads, head_dim)
        self.scales = None
        if scaled:
            each, blocks = math.prod(shape[3:]), page_size // (block or page_size)
            room = -(-blocks * kv_heads // 16) * 16
            pool = torch.zeros(layers, 2, pages, each + room, dtype=torch.uint8, device=device)
            self.data = pool[..., :each].view(shape)
            self.scales = pool[..., each:each + blocks * kv_heads].view(layers, 2, pages, blocks,
                                                                        kv_heads)
            self.pool = pool.flatten(0, 1)
        else:
            self.data = torch.zeros(shape, dtype=dtype, device=device)
            self.pool = self.data.flatten(0, 1)
        self.table = torch.full((rows, width), -1, **ints)
        self.lens = torch.zeros(rows, **ints)
        self.ws = attn.Workspace(device)
        # the tables are written from one into the other
        self._next = torch.empty_like(self.table), torch.empty_like(self.lens)

    def turn(self, rec, parent, room):
        """Row i becomes a continuation of row parent[i] (-1: empty) with room for
        room[i] tokens; pages in use move to the front of the pool."""
        table, lens = self._next
        ints = dict(dtype=torch.int32, device=self.table.device)
        rows, pages, entries = len(parent), self.pool.shape[1], table.numel()
        # a page in every plane, read and written
        each = self.pool.shape[0] * self.pool[0, 0].numel() * self.pool.element_size()
        lens_in, lens_out = self.lens.clone(), torch.empty_like(lens)

        def copied():
            """Bytes of the part-filled pages that the fork copied: those of rows
            that are not their parent's first, where the copy got a page."""
            had, has = lens_in.tolist(), lens_out.tolist()
            return each * sum(p >= 0 and p in parent[:i] and had[p] % self.page_size > 0
                              and has[i] == had[p] for i, p in enumerate(parent))

        def moved(out):
            to = out["moved"]
            return each * int(((to >= 0) & (to != torch.arange(pages, **ints))).sum())

        with rec.op("cache::turn"):
            rec.launch("pages_fork", lambda out: 4 * (entries + 3 * rows) + copied(),
                       lambda out: 4 * (entries + rows + pages) + copied(),
                       attn.opattr_pages_fork, self.pool, self.page_size, self.table, self.lens,
                       torch.tensor(parent, **ints), torch.tensor(room, **ints),
                       table_out=table, lens_out=lens, ws=self.ws)
            lens_out.copy_(lens)  # which later steps write again
            self._next = self.table, self.lens
            self.table, self.lens = table, lens
            out = rec.launch("pages_compact", lambda out: 4 * entries + moved(out),
                             lambda out: 4 * (entries + pages + 1) + moved(out),
                             attn.opattr_pages_compact, self.pool, table, table_out=table,
                             ws=self.ws)
        return out["live"]

    def append(self, rec, layer, k, v, cu, lens_out):
        size = 2 * k.numel() * k.element_size()
        with rec.op("cache::append"):
            if self.scales is not None:
                rec.launch("kv_append_scaled", size, 2 * k.numel(), attn.opattr_kv_append_scaled,
                           k, v, cu, *self.data[layer], *self.scales[layer], self.table,
                           self.lens, lens_out=lens_out)
            else:
                rec.launch("kv_append", size, size, attn.opattr_kv_append, k, v, cu,
                           self.data[layer, 0], self.data[layer, 1], self.table, self.lens,
                           lens_out=lens_out)

    def _blocks(self, n, window, sinks):
        """Blocks with one exponent of which a query that comes after n - 1 tokens sees a
        token."""
        block = self.page_size // self.scales.shape[3]
        first = 0 if window is None else max(0, n - window)
        blocks = -(-n // block) - first // block
        sinks = -(-min(sinks, first) // block)  # the last of them may be the window's first
        return blocks + min(sinks, first // block)

    def attend(self, rec, layer, q, lens, sizes, scale, window=None, sinks=0):
        """Attention of one token a sequence over the layer's cache, of the given
        lengths (on the device, and as numbers): (out, lse)."""
        seen = sum(n if window is None else min(n, window + min(sinks, max(0, n - window)))
                   for n in sizes)
        k, v = self.data[layer]
        rows = q.numel() * q.element_size()
        read = 2 * seen * k.shape[2] * k.shape[3] * k.element_size() + rows
        kw = dict(scale=scale, ws=self.ws)
        if self.scales is not None:
            read += 2 * k.shape[2] * sum(self._blocks(n, window, sinks) for n in sizes)
            return rec.launch("attn_paged_scaled", read, rows, attn.opattr_attn_paged_scaled, q, k,
                              v, *self.scales[layer], self.table, lens, window=window,
                              sinks=sinks, **kw)
        if window is not None:
            return rec.launch("attn_paged_window", read, rows, attn.opattr_attn_paged_window, q, k,
                              v, self.table, lens, window, sinks, **kw)
        return rec.launch("attn_paged", read, rows, attn.opattr_attn_paged, q, k, v, self.table,
                          lens, **kw)


def _rows(n, heads, kv_heads, head_dim, gen, dtype):
    rows = torch.randn(n, heads + 2 * kv_heads, head_dim, generator=gen, device="cuda:0").to(dtype)
    return rows[:, :heads], rows[:, heads:heads + kv_heads], rows[:, heads + kv_heads:]


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda:0")


def _starts(lens):
    return _ints([0, *np.cumsum(lens).tolist()])


def _prompt(rec, read, q, k, v, cu, window, sinks, **kw):
    written = q.numel() * q.element_size()
    if window is None:
        return rec.launch("attn_prompt", read, written, attn.opattr_attn_prompt, q, k, v, cu,
                          causal=True, **kw)
    return rec.launch("attn_prompt_window", read, written, attn.opattr_attn_prompt_window, q, k, v,
                      cu, window, sinks, **kw)


def serve(rec, lens=(100, 37, 64), steps=8, layers=2, heads=8, kv_heads=4, head_dim=64,
          page_size=16, dtype=torch.bfloat16, seed=0, window=None, sinks=0, scaled=False):
    """Prompts of the given lengths, `steps` tokens each, a turn in which the
    first sequence is forked into the place of the second, and `steps` more; through a
    window with sinks, if one is given, and from a cache of 8 bits, if scaled. Returns,
    for every sequence alive at the end, its layers' queries, keys, values and outputs,
    each [tokens, heads, head_dim]."""
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(seed)
    rows, most = len(lens), max(lens) + 2 * steps
    width = -(-most // page_size)
    cache = Cache(layers, 2 * rows * width, page_size, kv_heads, head_dim, rows, width, dtype,
                  scaled=scaled)
    cache.turn(rec, [-1] * rows, [n + steps for n in lens])
    history = [[[] for _ in range(layers)] for _ in range(rows)]
    sizes, cu, one = list(lens), _starts(lens), _starts([1] * rows)
    scale, each = 1 / math.sqrt(head_dim), head_dim * torch.finfo(dtype).bits // 8
    after = torch.empty_like(cache.lens)
    with rec.op("model::prompt"):
        for layer in range(layers):
            q, k, v = _rows(sum(lens), heads, kv_heads, head_dim, gen, dtype)
            with rec.op("aten::attention"):
                out, _ = _prompt(rec, (q.shape[0] * (heads + 2 * kv_heads)) * each, q, k, v, cu,
                                 window, sinks, scale=scale)
            cache.append(rec, layer, k, v, cu, after)
            for b in range(rows):
                s = slice(sum(lens[:b]), sum(lens[:b + 1]))
                history[b][layer].append((q[s], k[s], v[s], out[s]))
        cache.lens.copy_(after)

    def generate():
        for _ in range(steps):
            with rec.op("model::step"):
                for layer in range(layers):
                    q, k, v = _rows(rows, heads, kv_heads, head_dim, gen, dtype)
                    cache.append(rec, layer, k, v, one, after)
                    with rec.op("aten::attention"):
                        out, _ = cache.attend(rec, layer, q, after, [n + 1 for n in sizes], scale,
                                              window, sinks)
                    for b in range(rows):
                        s = slice(b, b + 1)
                        history[b][layer].append((q[s], k[s], v[s], out[s]))
                cache.lens.copy_(after)
                for b in range(rows):
                    sizes[b] += 1

    generate()
    parent = [0 if b == 1 else b for b in range(rows)]
    sizes[:] = [sizes[p] for p in parent]
    history = [[list(h) for h in history[p]] for p in parent]
    cache.turn(rec, parent, [n + steps for n in sizes])
    generate()
    return [[tuple(torch.cat(t) for t in zip(*h)) for h in seq] for seq in history]


def train(rec, lens=(300, 120, 77), heads=8, kv_heads=4, head_dim=64, dtype=torch.bfloat16,
          seed=0, window=None, sinks=0):
    """One attention layer over packed documents, forward and backward, through a window
    with sinks, if one is given. Returns the output and the gradients of queries, keys
    and values."""
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(seed)
    cu, n = _starts(lens), sum(lens)
    q, k, v = _rows(n, heads, kv_heads, head_dim, gen, dtype)
    dout = torch.randn(q.shape, generator=gen, device="cuda:0").to(dtype)
    each = head_dim * torch.finfo(dtype).bits // 8
    read = n * (heads + 2 * kv_heads) * each
    with rec.op("model::train"):
        with rec.op("aten::attention"):
            out, lse = _prompt(rec, read, q, k, v, cu, window, sinks)
        with rec.op("aten::attention_backward"):
            if window is None:
                grads = rec.launch("attn_prompt_grad", read + 2 * n * heads * each, read,
                                   attn.opattr_attn_prompt_grad, dout, q, k, v, out, lse, cu)
            else:
                grads = rec.launch("attn_prompt_window_grad", read + 2 * n * heads * each, read,
                                   attn.opattr_attn_prompt_window_grad, dout, q, k, v, out, lse,
                                   cu, window, sinks)
    return (out, *grads)


def main(argv):
    parser = argparse.ArgumentParser(description=__doc__, prog="workload",
                                     formatter_class=argparse.RawDescriptionHelpFormatter)
    parser.add_argument("profile", help="the profile document that is written")
    parser.add_argument("--window", type=int, help="tokens of a sliding window")
    parser.add_argument("--sinks", type=int, default=0, help="first tokens that stay visible")
    parser.add_argument("--scaled", action="store_true", help="a cache of 8 bits")
    args = parser.parse_args(argv[1:])
    window = dict(window=args.window, sinks=args.sinks)
    for rec in (Recorder(), Recorder()):  # the first loads the kernels
        serve(rec, scaled=args.scaled, **window)
        train(rec, **window)
    doc = profile(rec)
    profile_doc.write(args.profile, doc)
    total = {}
    for entry in doc["operators"]:
        t = total.setdefault(entry["operator_name"], [0, 0, 0.0])
        t[0] += 1
        t[1] += entry["aggregated"]["total_duration_ns"]
        t[2] += entry["aggregated"]["dram_bytes_read"] + entry["aggregated"]["dram_bytes_written"]
    for name, (calls, ns, moved) in sorted(total.items(), key=lambda x: -x[1][1]):
        print(f"{name:28s} {calls:4d} dispatches {ns / 1e3:10.1f} us {moved / 1e6:10.2f} MB")
    return 0


if __name__ == "__main__":
    sys.exit(main(sys.argv))
