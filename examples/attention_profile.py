"""A small serving loop, profiled by the library itself.

One attention layer (12 heads of 64) serves a few chats: their prompts go through
Context.attention and into a paged cache, then every chat grows token by token
(cache_append, cache_attention), one is forked into two continuations, some end
(cache_trim) and the cache is compacted.  Every launch is timed, and what is known of
its traffic stands in for the Nsight Compute rows; the join attributes both to the
calls, rolls them up by operator and writes profile.json.

    python examples/attention_profile.py [profile.json]
"""
from __future__ import annotations

import os
import sys
import time

import numpy as np
import torch

if __name__ == "__main__":
    sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2609_11938_gb300 as opa  # noqa: E402

HEADS, DIM, PAGE = 12, 64, 16
ROW = HEADS * DIM * 2                    # bytes of a token's keys, or values, or queries
OPERATORS = ["aten::attention", "aten::cache_append", "aten::cache_attention", "aten::cache_fork", "aten::cache_trim",
             "aten::cache_compact"]
TIME, READ, WRITTEN = 0, 1, 2            # columns of the counters that are known


class Recorder:
    """Calls as operator ranges, their launches as kernel records with a row each."""

    def __init__(self, ctx):
        self.ctx, self.names, self.ranges, self.kernels, self.rows = ctx, [], [], [], []
        ctx.set_timing(True)

    def call(self, operator: int, mover: str, read: int, written: int, run):
        """Runs one call; `mover` is the kernel that moves its data."""
        self.ctx.timing_reset()
        start = time.perf_counter_ns()
        result = run()
        self.ctx.check()
        at = start
        for name, (ms, launches) in self.ctx.timing_report().items():
            for _ in range(launches):
                if name not in self.names:
                    self.names.append(name)
                ns = max(1, round(1e6 * ms / launches))
                at += 1
                self.kernels.append((at, ns, self.names.index(name)))
                row = np.full(opa.N_COUNTERS, np.nan, np.float32)
                row[TIME], row[READ], row[WRITTEN] = ns, read if name == mover else 0, written if name == mover else 0
                self.rows.append(row)
        self.ranges.append((start, max(time.perf_counter_ns(), at + 1), operator))
        return result

    def trace(self) -> opa.DeviceTrace:
        dev = f"cuda:{self.ctx.device}"
        k, r = np.array(self.kernels, np.int64), np.array(self.ranges, np.int64)
        up = lambda a, dt: torch.from_numpy(np.ascontiguousarray(a, dtype=dt)).to(dev)  # noqa: E731
        name = up(k[:, 2], np.int32)
        return opa.DeviceTrace(up(np.zeros(len(k)), np.uint8), up(k[:, 0], np.int64), up(k[:, 1], np.int64), name, None,
                               up(np.zeros(len(r)), np.uint8), up(r[:, 0], np.int64), up(r[:, 1], np.int64),
                               up(np.zeros(len(r)), np.uint8), up(np.arange(len(r)), np.int32), len(r), name,
                               up(np.stack(self.rows), np.float32))


def serve(rec: Recorder, prompts=(128, 70, 200, 33), steps=8, seed=0):
    """The serving loop.  Returns the cache and the last step's queries and results."""
    ctx = rec.ctx
    dev = f"cuda:{ctx.device}"
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    new = lambda n: [torch.randn((n, HEADS, DIM), generator=gen, device=dev).bfloat16() for _ in range(3)]  # noqa: E731
    i32 = lambda x: torch.tensor(list(x), dtype=torch.int32, device=dev)  # noqa: E731
    n_seqs, per_seq = len(prompts) + 2, -(-(max(prompts) + steps + 8) // PAGE)
    cache = ctx.cache(n_seqs * per_seq, PAGE, HEADS, DIM, n_seqs, per_seq)
    lengths = list(prompts) + [0, 0]
    # prompts
    tokens = sum(prompts)
    offsets = i32(np.concatenate([[0], np.cumsum(prompts)]))
    q, k, v = new(tokens)
    rec.call(0, "prompt", 3 * ROW * tokens, ROW * tokens, lambda: ctx.attention(q, k, v, offsets))
    rec.call(1, "append_rows", 2 * ROW * tokens, 2 * ROW * tokens,
             lambda: ctx.cache_append(cache, i32(range(len(prompts))), offsets, k, v))
    live = list(range(len(prompts)))
    q = out = None

    def step():
        nonlocal q, out
        n = len(live)
        seqs = i32(live)
        q, k, v = new(n)
        rec.call(1, "append_rows", 2 * ROW * n, 2 * ROW * n, lambda: ctx.cache_append(cache, seqs, i32(range(n + 1)), k, v))
        for s in live:
            lengths[s] += 1
        seen = sum(lengths[s] for s in live)
        out = rec.call(2, "token", 2 * ROW * seen + ROW * n, ROW * n, lambda: ctx.cache_attention(cache, seqs, q)[1])

    for _ in range(steps):
        step()
    # two continuations of the first chat beside it
    rec.call(3, "fork_plan", 0, 0, lambda: ctx.cache_fork(cache, i32([0, 0]), i32([n_seqs - 2, n_seqs - 1])))
    lengths[n_seqs - 2] = lengths[n_seqs - 1] = lengths[0]
    live += [n_seqs - 2, n_seqs - 1]
    step()
    # two chats end, and the pages move together
    for s in (1, n_seqs - 2):
        live.remove(s)
        lengths[s] = 0
    rec.call(4, "trim_plan", 0, 0, lambda: ctx.cache_trim(cache, i32([1, n_seqs - 2])))
    used = cache.refs > 0
    moved = int(used[int(used.sum()):].sum())
    rec.call(5, "compact_move", 2 * ROW * PAGE * moved, 2 * ROW * PAGE * moved, lambda: ctx.cache_compact(cache))
    step()
    return cache, live, q, out


def profile(rec: Recorder, path):
    """Joins what was recorded; writes profile.json and returns per-operator records."""
    ctx = rec.ctx
    ctx.set_timing(False)
    tr = rec.trace()
    _, out, ops, matched, totals = ctx.join(tr)
    of = np.array([r[2] for r in rec.ranges], np.int32)
    _, rolled = ctx.rollup(tr, out["range_of_kernel"], out["ncu_idx"], torch.from_numpy(of).to(tr.k_start.device),
                           len(OPERATORS))
    host = lambda d: {k: x.cpu().numpy() for k, x in d.items()}  # noqa: E731
    opa.write_profile(path, tr.k_stream.cpu().numpy(), tr.k_dur.cpu().numpy(), tr.k_name.cpu().numpy(),
                      out["range_of_kernel"].cpu().numpy().view(np.uint32), out["ncu_idx"].cpu().numpy(),
                      tr.counters.cpu().numpy(), host(ops), kernel_names=rec.names,
                      op_names=[OPERATORS[i] for i in of],
                      meta={"model_name": "attention layer, 12 heads of 64", "device_name": torch.cuda.get_device_name(),
                            "compile_mode": "eager"})
    return host(rolled), matched, totals


def main(path="profile.json"):
    with opa.Context(0) as ctx:
        rec = Recorder(ctx)
        serve(Recorder(ctx))                             # code is loaded and scratch made once, untimed
        serve(rec)
        rolled, matched, totals = profile(rec, path)
    print(f"{'operator':24s} {'launches':>8s} {'us':>9s} {'MB read':>9s} {'MB written':>10s} {'GB/s':>7s}")
    for i, name in enumerate(OPERATORS):
        ns, read, written = rolled["total_duration_ns"][i], rolled["agg"][READ, i], rolled["agg"][WRITTEN, i]
        print(f"{name:24s} {rolled['kernel_count'][i]:8d} {ns / 1e3:9.1f} {read / 1e6:9.2f} {written / 1e6:10.2f} "
              f"{(read + written) / ns:7.1f}")
    print(f"{totals['attributed_kernels']} of {totals['kernels']} launches attributed, {matched['direct']} with a row; "
          f"{path} written")
    return rolled, matched, totals


if __name__ == "__main__":
    main(*sys.argv[1:2])
