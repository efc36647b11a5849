"""A serving node's paged cache in plain Python and 64-bit NumPy, from the rules
of include/agft_kv.h: what the GPU tests compare with.  One request, one token,
one page at a time; no code shared with the package."""
import math

import numpy as np

RANGE = {"e4m3": 448.0, "int8": 127.0}
E_MIN = -64


def exponent(top, form):
    """The smallest e >= E_MIN with top <= range * 2^e."""
    e = E_MIN
    if top > RANGE[form] * 2.0 ** E_MIN:
        e = math.floor(math.log2(top / RANGE[form])) - 1
        while top > RANGE[form] * 2.0 ** e:
            e += 1
    return max(e, E_MIN)


def held(y, form):
    """y (already divided by 2^e) as the code stands for it."""
    y = np.where(np.isnan(y), 0.0, np.clip(y, -RANGE[form], RANGE[form]))
    if form == "int8":
        return np.rint(y)
    _, x = np.frexp(y)
    quantum = 2.0 ** (np.maximum(x - 1, -6) - 3)
    return np.rint(y / quantum) * quantum


class Node:
    """Tables and one layer's cache."""

    def __init__(self, requests, row_pages, pages, page, heads, group, dim, form):
        self.R, self.W, self.P, self.page = requests, row_pages, pages, page
        self.H, self.G, self.D, self.form = heads, group, dim, form
        self.lengths = [0] * requests
        self.table = np.zeros((requests, row_pages), dtype=np.int64)
        self.ring = list(range(pages))
        self.head, self.free = 0, pages
        self.codes = np.zeros((pages, heads, 2, page, dim))
        self.exps = np.zeros((pages, heads, 2), dtype=np.int64)

    def _pages(self, n):
        return -(-n // self.page)

    def plan(self, add, max_tokens):
        """The window's parts as a dict; lengths and counters change at commit."""
        starts, granted, lengths, slots = [0], [], [], [-1] * max_tokens
        at = cum = taken = refused = gone = 0
        table = self.table.copy()
        for i, a in enumerate(add):
            past = self.lengths[i]
            have = self._pages(past)
            ask = a if a > 0 and past + a <= self.W * self.page else 0
            need = self._pages(past + ask) - have
            base = cum
            cum += need
            ok = ask > 0 and (need == 0 or cum <= self.free) and at + ask <= max_tokens
            if ok:
                taken += need
                for n in range(need):
                    table[i, have + n] = self.ring[(self.head + base + n) % self.P]
                for k in range(ask):
                    t = past + k
                    slots[at + k] = int(table[i, t // self.page]) * self.page + t % self.page
            if a < 0:
                for n in range(have):
                    self.ring[(self.head + self.free + gone) % self.P] = int(self.table[i, n])
                    gone += 1
            refused += a > 0 and not ok
            granted.append(ask if ok else 0)
            lengths.append(0 if a < 0 else past + granted[-1])
            at += ask
            starts.append(min(at, max_tokens))
        self.table = table
        return dict(starts=starts, granted=granted, lengths=lengths, slots=slots,
                    counters=[(self.head + taken) % self.P, self.free - taken + gone, starts[-1], refused, taken, gone,
                              0, 0])

    def commit(self, step):
        self.lengths = list(step["lengths"])
        self.head, self.free = step["counters"][:2]

    def append(self, step, k, v):
        """k, v [tokens][heads][dim], 64 bits."""
        runs = {}
        for t, slot in enumerate(step["slots"]):
            if slot >= 0:
                runs.setdefault(slot // self.page, []).append((t, slot % self.page))
        for page, tokens in runs.items():
            rows, offs = [t for t, _ in tokens], [o for _, o in tokens]
            for h in range(self.H):
                for side, x in enumerate((k, v)):
                    new = x[rows, h]
                    finite = np.abs(new[np.isfinite(new)])
                    e = exponent(finite.max() if finite.size else 0.0, self.form)
                    if offs[0] > 0:
                        old = int(self.exps[page, h, side])
                        e = max(e, old)
                        if e > old:
                            self.codes[page, h, side] = held(self.codes[page, h, side] * 2.0 ** (old - e), self.form)
                    self.exps[page, h, side] = e
                    self.codes[page, h, side][offs] = held(new * 2.0 ** -float(e), self.form)

    def export(self, slots):
        """Values [n][heads][2][dim] of the slots."""
        out = np.zeros((len(slots), self.H, 2, self.D))
        for n, s in enumerate(slots):
            if s >= 0:
                p, o = s // self.page, s % self.page
                out[n] = self.codes[p, :, :, o] * (2.0 ** self.exps[p].astype(float))[..., None]
        return out

    def attend(self, step, q, scale):
        """q [tokens][heads * group][dim], 64 bits.  Returns out, lse, and per
        row the largest |v|, the largest sum of |q k| scale, and the keys."""
        n_rows = step["starts"][-1]
        HQ = self.H * self.G
        out = np.zeros((n_rows, HQ, self.D))
        lse = np.full((n_rows, HQ), -np.inf)
        vmax, smax, keys = np.zeros((n_rows, HQ)), np.zeros((n_rows, HQ)), np.zeros((n_rows, HQ))
        for i in range(self.R):
            n = step["granted"][i]
            if not n:
                continue
            L = step["lengths"][i]
            kv = self.export([int(self.table[i, t // self.page]) * self.page + t % self.page for t in range(L)])
            for j in range(n):
                row, m = step["starts"][i] + j, L - n + j + 1
                for h in range(self.H):
                    k, v = kv[:m, h, 0], kv[:m, h, 1]
                    for g in range(self.G):
                        x = q[row, h * self.G + g]
                        s = k @ x * scale
                        top = s.max()
                        p = np.exp(s - top)
                        out[row, h * self.G + g] = p @ v / p.sum()
                        lse[row, h * self.G + g] = top + np.log(p.sum())
                        vmax[row, h * self.G + g] = np.abs(v).max()
                        smax[row, h * self.G + g] = (np.abs(k) @ np.abs(x)).max() * abs(scale)
                        keys[row, h * self.G + g] = m
        return out, lse, vmax, smax, keys
