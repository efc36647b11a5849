"""Attention over a paged cache whose codes are given, in 64 bits, and how far
from it a right kernel may be.  For data that shows what an attention sums: no
key outweighs the others by much, or by exactly as much as a test wants.

The bound.  With u the largest share that rounding to the output's type takes
(2^-8 bf16, 2^-11 fp16: half a step of 8 or 11 bits, beside a number just above
a power of two), w_j the weights of the softmax and A = sum w_j |v_j|, an output is off by

    u |o| + z                       its own rounding, z = 2^-25 fp16's below 2^-14
    2^-11 A                         the probabilities' rounding to fp16
    2 e A, e = (D + 4) 2^-24 smax + 2^-23 (1.45 smax + |ev| + 64)
                                    a score's products and sums in fp32 and its
                                    scaling, twice (over the quotient); smax is
                                    the largest sum |q_d k_d| scale
    2 (N / 16 + 32) 2^-24 A         sums of N keys, 16 at a time, and joins, in fp32
    N 2^-32 max(w_j 2^ev_j) cmax    what fp16 loses of a probability 2^-32 below
                                    the largest, cmax the largest |code|

and the logarithm of the sum by e, the sums' part, and 2^-22 of its size."""
import math

import torch

from paper_2508_01744_amd import KvCache, KvTables, kv_config

T = {"bf16": torch.bfloat16, "fp16": torch.float16}
E4M3 = [(-1.0 if c & 128 else 1.0) * (math.nan if c & 127 == 127 else (c & 7) * 2.0 ** -9 if c & 120 == 0 else
                                     (8 + (c & 7)) * 2.0 ** (((c >> 3) & 15) - 10)) for c in range(256)]
INT8 = [float(c if c < 128 else c - 256) for c in range(256)]


class Window:
    """Requests of `past` tokens that bring `add` more, over pages of random
    codes in a random order: keys of either sign, values positive, magnitudes
    within a factor of four and, for values, another factor of up to eight from
    page to page, so that every page's share of a sum is its own."""

    def __init__(self, past, add, page, heads, group, dim, form, dtype, seed, device="cuda"):
        self.past, self.add, self.page, self.heads, self.group, self.dim = past, add, page, heads, group, dim
        self.form, self.dtype, self.device = form, T[dtype], device
        gen = torch.Generator(device=device).manual_seed(seed)
        held = [-(-p // page) for p in past]
        all_pages = [-(-(p + max(a, 0)) // page) for p, a in zip(past, add)]
        self.pages, self.row_pages = sum(all_pages), max(1, max(all_pages))
        order = torch.randperm(self.pages, generator=gen, device=device).tolist()
        self.rows, at, fresh = [], 0, sum(held)
        for h, n in zip(held, all_pages):
            self.rows.append(order[at:at + h] + order[fresh:fresh + n - h])
            at, fresh = at + h, fresh + n - h
        self.held, self.free = held, order[sum(held):]
        shape = (self.pages, heads, 2, page, dim)
        if form == "e4m3":
            codes = torch.randint(0x30, 0x40, shape, generator=gen, device=device, dtype=torch.int16)    # 0.5 .. 1.875
            codes[:, :, 0] |= 128 * torch.randint(0, 2, (self.pages, heads, page, dim), generator=gen, device=device,
                                                  dtype=torch.int16)
            unit = 0
        else:
            codes = torch.randint(32, 121, shape, generator=gen, device=device, dtype=torch.int16)
            codes[:, :, 0] *= 1 - 2 * torch.randint(0, 2, (self.pages, heads, page, dim), generator=gen, device=device,
                                                    dtype=torch.int16)
            unit = -6
        self.codes = (codes & 255).to(torch.uint8)
        self.exps = torch.stack([torch.randint(unit - 1, unit + 1, (self.pages, heads), generator=gen, device=device),
                                 torch.randint(unit - 2, unit + 2, (self.pages, heads), generator=gen, device=device)],
                                2).to(torch.int32)
        self.tokens = sum(max(a, 0) for a in add)
        # scores of about +-1
        q = torch.randn(self.tokens, heads * group, dim, generator=gen, device=device) * 0.7
        self.q = q.to(self.dtype)
        self.scale = 1.0 / math.sqrt(dim)

    def on_gpu(self, max_new=None):
        """The package's tables, cache and planned step, loaded with this."""
        cfg = kv_config(len(self.past), self.row_pages * self.page, self.pages, page=self.page, heads=self.heads,
                        group=self.group, dim=self.dim, form=self.form)
        tables, cache = KvTables(cfg), KvCache(cfg)
        table = torch.zeros(len(self.past), self.row_pages, dtype=torch.int32)
        for i, (row, h) in enumerate(zip(self.rows, self.held)):
            table[i, :h] = torch.tensor(row[:h], dtype=torch.int32)
        ints = lambda x: torch.tensor(x, dtype=torch.int32, device=self.device)         # noqa: E731
        tables.load(ints(self.past), table.to(self.device), ints(self.free))
        cache.load(self.codes, self.exps)
        step = tables.plan(ints(self.add), self.tokens, max_new=max_new or max(1, max(self.add)))
        return tables, cache, step

    def reference(self, spoil=None):
        """out, lse in 64 bits, and the bounds on how far each may be off.
        spoil(weights [rows][L], v [L][dim], at): changes a copy of a request's
        unnormalised weights of the products, for tests of the bound itself."""
        values = torch.tensor(E4M3 if self.form == "e4m3" else INT8, dtype=torch.float64, device=self.device)
        H, G, D = self.heads, self.group, self.dim
        out = torch.zeros(self.tokens, H * G, D, dtype=torch.float64, device=self.device)
        lse, room = torch.zeros_like(out[..., 0]), torch.zeros_like(out)
        lse_room = torch.zeros_like(lse)
        u, z = (2.0 ** -8, 0.0) if self.dtype == torch.bfloat16 else (2.0 ** -11, 2.0 ** -25)
        first = 0
        for past, n, row in zip(self.past, self.add, self.rows):
            if n <= 0:
                continue
            N = past + n
            ids = torch.tensor(row, device=self.device)
            last = past + torch.arange(n, device=self.device).repeat_interleave(G)
            hidden = torch.arange(N, device=self.device)[None, :] > last[:, None]
            for h in range(H):
                code = values[self.codes[ids, h].long()]                               # [pages][2][page][D]
                e = self.exps[ids, h].double()
                kv = code * torch.exp2(e)[..., None, None]
                k, v = (kv[:, s].reshape(-1, D)[:N].contiguous() for s in (0, 1))
                q = self.q[first:first + n, h * G:(h + 1) * G].double().reshape(n * G, D)
                s = (q @ k.t().contiguous()) * self.scale
                s.masked_fill_(hidden, -math.inf)
                smax = ((q.abs() @ k.abs().t().contiguous()) * self.scale).masked_fill_(hidden, 0).amax(1)
                w = torch.softmax(s, 1)
                into = w if spoil is None else spoil(w.clone(), v, past)
                o = into @ v
                total = torch.logsumexp(s, 1)
                A = w @ v.abs()
                ev = e[:, 1].repeat_interleave(self.page)[:N]
                off = (D + 4) * 2.0 ** -24 * smax + 2.0 ** -23 * (1.45 * smax + ev.abs().max() + 64)
                sums = 2 * (N / 16 + 32) * 2.0 ** -24
                gone = N * 2.0 ** -32 * (w * torch.exp2(ev)).amax(1) * code[:, 1].abs().max()
                tol = u * (w @ v).abs() + (2.0 ** -11 + 2 * off + sums)[:, None] * A + gone[:, None] + z + 2.0 ** -40
                at, heads = slice(first, first + n), slice(h * G, (h + 1) * G)
                out[at, heads], room[at, heads] = o.view(n, G, D), tol.view(n, G, D)
                lse[at, heads] = total.view(n, G)
                lse_room[at, heads] = (off + sums + 2.0 ** -22 * (1 + total.abs())).view(n, G)
            first += n
        return out, lse, room, lse_room


def compare(window, max_new=None, tell=""):
    """The kernels on this window against the reference; the largest share of
    the bound that an output takes."""
    tables, cache, step = window.on_gpu(max_new)
    shape = (window.tokens, window.heads * window.group)
    lse = torch.full(shape, 7.0, device=window.device)
    out = cache.attend(tables, step, window.q, lse=lse, scale=window.scale)
    ref, ref_lse, room, lse_room = window.reference()
    share = ((out.double() - ref).abs() / room)
    lse_share = ((lse.double() - ref_lse).abs() / lse_room)
    worst, worst_lse = float(share.max()), float(lse_share.max())
    print("  ", tell, "worst share of the bound", worst, "of the logarithm's", worst_lse, flush=True)
    assert bool((share <= 1).all()), (tell, worst, torch.nonzero(share > 1)[:4].tolist())
    assert bool((lse_share <= 1).all()), (tell, worst_lse, torch.nonzero(lse_share > 1)[:4].tolist())
    return tables, cache, step
