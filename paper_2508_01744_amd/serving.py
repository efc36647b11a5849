"""A serving node whose window is measured instead of computed: requests from a
workload's load trace hold pages of an 8-bit cache (KvTables, KvCache) and go
through the window's cache and attention work, layer by layer, and a tuner sees
the node that results (Sec. 4.1's collector, features and decision loop, Fig. 5).

What is real: continuous batching of prompts (in chunks) and single tokens,
block tables, cache writes, attention, and their time, from the first call to
the end of the work on the GPU: a window of little work takes as long as the
host needs for its calls (4 to 8 us each).  What is not: the
numbers (queries, keys and values are drawn once), the rest of a model, and the
clock: the card's own stays as it is.  A decision's clock f enters by the closed
form that the simulator uses, power P0 + c f^3 and a latency of which the share
`a` does not depend on it:

    latency = (a + (1 - a) f_hi / f) * (measured time per token) / (its running mean)
    reward  = -power(f) latency^2 / power(f_hi)

    python -m paper_2508_01744_amd.serving --windows 300 [--layers 4] [--form int8]
"""
import argparse
import json
import math
import sys

import numpy as np
import torch

from agft_workloads import ENV, arm_values, exogenous, get_workload
from .kv import KvCache, KvStep, KvTables, kv_config
from .tuner import Tuner


class Batch:
    """Continuous batching on the host: which request holds which row of the
    block table, and how many new tokens each brings to a window."""

    def __init__(self, rows, queue_cap, tokens, row_tokens, seed=0):
        if rows < 1 or tokens < 1 or row_tokens < 32:
            raise ValueError("a node has at least one row of 32 tokens or more, and windows of a token or more")
        self.rows, self.queue_cap, self.tokens, self.row_tokens = rows, queue_cap, tokens, row_tokens
        self.rng = np.random.default_rng(seed)
        self.queue = []                     # (prompt, outputs) of requests that wait
        self.left = [None] * rows           # [prompt tokens to bring, tokens to make] of running ones
        self.ended = [False] * rows         # rows whose pages go back in the next window
        self.dropped = self.served = 0

    def _request(self):
        prompt, outputs = (int(round(math.exp(self.rng.uniform(math.log(lo), math.log(hi)))))
                           for lo, hi in ((16, self.row_tokens // 2), (4, self.row_tokens // 8)))
        return [prompt, outputs]

    @property
    def running(self):
        return sum(x is not None for x in self.left)

    def window(self, arrivals):
        """New tokens per row (-1: the request ended in the last window)."""
        for _ in range(arrivals):
            if len(self.queue) < self.queue_cap:
                self.queue.append(self._request())
            else:
                self.dropped += 1
        add = [0] * self.rows
        budget = self.tokens
        for i in range(self.rows):
            if self.ended[i]:
                add[i], self.ended[i] = -1, False
            elif self.left[i] is None and self.queue:
                self.left[i] = self.queue.pop(0)
        # the next token of requests past their prompt first, then prompts in chunks
        for i, x in enumerate(self.left):
            if x is not None and x[0] == 0 and budget > 0 and add[i] == 0:
                add[i], budget = 1, budget - 1
        for i, x in enumerate(self.left):
            if x is not None and x[0] > 0 and budget > 0 and add[i] == 0:
                add[i] = min(x[0], budget)
                budget -= add[i]
        for i, x in enumerate(self.left):
            if x is None or add[i] <= 0:
                continue
            if x[0] > 0:
                x[0] -= add[i]
            else:
                x[1] -= 1
                if x[1] == 0:
                    self.left[i], self.ended[i] = None, True
                    self.served += 1
        return add


class ServingNode:
    """The node: tables, one cache per layer, and a window's work."""

    def __init__(self, layers=2, rows=64, row_tokens=4096, tokens=1024, page=16, heads=8, group=4, dim=128,
                 form="e4m3", dtype=torch.bfloat16, device="cuda", seed=0):
        pages = rows * -(-row_tokens // page)       # (every row can grow to its end: nothing is refused)
        self.cfg = kv_config(rows, row_tokens, pages, page=page, heads=heads, group=group, dim=dim, form=form)
        self.tables = KvTables(self.cfg, device)
        self.device = self.tables.device
        self.caches = [KvCache(self.cfg, self.device) for _ in range(layers)]
        self.step = KvStep(self.cfg, tokens, device=self.device)
        self.tokens = tokens
        gen = torch.Generator(device=self.device).manual_seed(seed)
        wide = torch.randn(tokens, (heads * group + 2 * heads) * dim, generator=gen, device=self.device).to(dtype)
        q, k, v = wide.split([heads * group * dim, heads * dim, heads * dim], 1)
        self.q, self.k, self.v = (x.unflatten(1, (-1, dim)) for x in (q, k, v))
        self.out = torch.empty(tokens, heads * group, dim, dtype=dtype, device=self.device)
        self._times = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)

    def window(self, add):
        """One window's work; the time in milliseconds from its first call to its
        end on the GPU, the host's time for the calls included where the GPU waits
        for them."""
        new = torch.tensor(add, dtype=torch.int32).to(self.device)
        first, last = self._times
        first.record()
        self.tables.plan(new, self.tokens, max_new=max(1, max(add)), step=self.step)
        for cache in self.caches:
            cache.append(self.step, self.k, self.v)
            cache.attend(self.tables, self.step, self.q, out=self.out)
        self.tables.commit(self.step)
        last.record()
        last.synchronize()
        return first.elapsed_time(last)


def features(arrivals, queue, running, latency, rows, used, clock):
    """The context of Sec. 4.1's stand-in, z-scored like the simulator's."""
    raw = (arrivals, math.log1p(queue), running, math.log(latency * (1.0 + queue / rows)), latency / ENV["tpot_div"],
           used, clock)
    return [1.0] + [(x - m) / s for x, m, s in zip(raw, ENV["mu"], ENV["sd"])]


def run(windows=300, workload="cfg1", seed=0, **node_options):
    """Let one tuner run a measured node for some windows; a summary dict."""
    if windows < 1:
        raise ValueError("at least one window")
    wl = get_workload(workload, B=1, T=windows)
    if wl.d != 8:
        raise ValueError("the measured node's context has 8 features")
    node = ServingNode(seed=seed, **node_options)
    cfg = node.cfg
    batch = Batch(cfg.requests, ENV["q_cap"], node.tokens, cfg.row_pages * cfg.page, seed)
    tuner = Tuner.from_workload(wl, device=node.device)
    arrivals = exogenous(wl)[0][:, 0]
    clocks = arm_values(wl.K)
    clock, reward, mean = ENV["f_init"], None, None
    action = torch.empty(1, dtype=torch.int32, device=node.device)
    chosen, times, tokens = [], [], 0
    for w in range(windows):
        add = batch.window(int(arrivals[w]))
        new = sum(a for a in add if a > 0)
        ms = node.window(add)
        if new:
            mean = ms / new if mean is None else 0.9 * mean + 0.1 * ms / new
        share = ENV["a"]
        latency = max(ENV["lat_min"], (share + (1 - share) * ENV["f_hi"] / clock) * (ms / new / mean if new else 1.0))
        power = ENV["P0"] + ENV["c"] * clock ** 3
        if w:
            reward = torch.tensor([-power * latency ** 2 / (ENV["P0"] + ENV["c"] * ENV["f_hi"] ** 3)],
                                  device=node.device)
        used = 1.0 - int(node.step.counters[1]) / cfg.pages
        ctx = torch.tensor([features(int(arrivals[w]), len(batch.queue), batch.running, latency, cfg.requests, used, clock)],
                           device=node.device)
        k = int(tuner.step(ctx, reward, action)[0])
        clock = clocks[k]
        chosen.append(k)
        times.append(ms)
        tokens += new
    times.sort()
    return dict(windows=windows, tokens=tokens, served=batch.served, dropped=batch.dropped, running=batch.running,
                queued=len(batch.queue), pages_used=used, window_ms_median=times[len(times) // 2],
                tokens_per_s=tokens / (sum(times) * 1e-3), arms_last_quarter=np.bincount(
                    chosen[-max(1, windows // 4):], minlength=wl.K).tolist())


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--windows", type=int, default=300)
    ap.add_argument("--workload", default="cfg1", help="load trace and arms; a workload with 8 features")
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--form", choices=("e4m3", "int8"), default="e4m3")
    ap.add_argument("--seed", type=int, default=0)
    args = ap.parse_args(argv)
    print(json.dumps(run(args.windows, args.workload, args.seed, layers=args.layers, form=args.form)))


if __name__ == "__main__":
    sys.exit(main())
