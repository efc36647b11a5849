"""The half of a differential attention's outputs whose values have the smaller scale, in
64 bits and relative to itself: how far from it a right kernel may be.

Each pair's second head has value exponents `apart` below the first head's, page by
page, and codes of its own (`windows`); the outputs are those of its dim numbers, 2^apart
times as large (gain), so that they are numbers of the outputs' types' middle range.

The bound.  With the pair's larger exponents e_j, codes c_j of the smaller half, weights
w_j of a map's softmax and, for each number, A = 2^-apart sum_j w_j 2^e_j |c_j|:

    2^-11 A                              the probabilities' rounding to fp16
    (2 e + sums) A                       scores, and sums in fp32: kv_flat's
    2^-32 max_j(w_j 2^e_j) 2^-apart sum_j |c_j|
                                         what fp16 loses of a probability, 2^-25 of one that is
                                         2^7 or more at the largest; relative to the larger
                                         scale, so it meets the smaller half times 2^-apart

and no more: the codes come to fp16 times 2^(lift - apart), and are whole there while their
smallest step, 2^-9 (e4m3) or 1 (int8), comes to 2^-24 or more: apart <= 22, 29.  Of the two
maps' difference y = y_0 - lambda y_1 and its factor in fp32 2^-22 (A_0 + |lambda| A_1), and
of the output u |out| + z (kv_flat's)."""
import math

import torch

from kv_flat import E4M3, INT8, Window

MOST = {"e4m3": 22, "int8": 29}
LIFT = {"e4m3": 7, "int8": 5}
# codes of the smaller half: the smallest numbers (which lose bits first), the largest, and all of them
CODES = {"small": (1, 16), "large": (0x70, 0x7F), "all": (0, 0x7F)}


def window(past, add, dim, form, dtype, apart, codes, seed, device="cuda", page=16):
    w = Window(past, add, page, 4, 2, dim, form, dtype, seed, device=device)
    w.exps[:, 1::2, 1] = w.exps[:, 0::2, 1] - apart
    gen = torch.Generator(device=device).manual_seed(seed + 1)
    shape = (w.pages, 2, page, dim)
    new = torch.randint(*CODES[codes], shape, generator=gen, device=device, dtype=torch.int16)
    if codes == "all":                                      # of either sign
        sign = torch.randint(0, 2, shape, generator=gen, device=device, dtype=torch.int16)
        new = new + 128 * sign if form == "e4m3" else new * (1 - 2 * sign)
    w.codes[:, 1::2, 1] = (new & 255).to(torch.uint8)
    return w


def lambdas(w, seed=0):
    gen = torch.Generator(device=w.device).manual_seed(seed)
    return torch.rand(w.heads // 2 * w.group, generator=gen, device=w.device) * 0.4 - 0.1


def smaller_half(w, lam, apart, spoil=None):
    """The second head's numbers, 2^apart times, and the bound.  spoil(c [N][dim]): a mistake in the codes' numbers."""
    values = torch.tensor(E4M3 if w.form == "e4m3" else INT8, dtype=torch.float64, device=w.device)
    G, D, pairs = w.group, w.dim, w.heads // 2
    out = torch.zeros(w.tokens, pairs * G, D, dtype=torch.float64, device=w.device)
    room = torch.zeros_like(out)
    u, z = (2.0 ** -8, 0.0) if w.dtype == torch.bfloat16 else (2.0 ** -11, 2.0 ** -25)
    first = 0
    for past, n, row in zip(w.past, w.add, w.rows):
        N, at = past + n, slice(first, first + n)
        ids = torch.tensor(row, device=w.device)
        last = past + torch.arange(n, device=w.device).repeat_interleave(G)
        hidden = torch.arange(N, device=w.device)[None, :] > last[:, None]
        for p in range(pairs):
            c = values[w.codes[ids, 2 * p + 1, 1].long()].reshape(-1, D)[:N]
            if spoil is not None:
                c = spoil(c)
            e = w.exps[ids, 2 * p, 1].double().repeat_interleave(w.page)[:N]
            y, d, total, heads = 0.0, 0.0, 0.0, slice(p * G, (p + 1) * G)
            la = lam[heads].double().repeat(n)[:, None]
            for a in (0, 1):
                k = values[w.codes[ids, 2 * p + a, 0].long()] * torch.exp2(w.exps[ids, 2 * p + a, 0].double())[:, None, None]
                k = k.reshape(-1, D)[:N].contiguous()
                q = w.q[at, (2 * p + a) * G:(2 * p + a + 1) * G].double().reshape(n * G, D)
                s = ((q @ k.t().contiguous()) * w.scale).masked_fill_(hidden, -math.inf)
                smax = ((q.abs() @ k.abs().t().contiguous()) * w.scale).masked_fill_(hidden, 0).amax(1)
                x = torch.softmax(s, 1) * torch.exp2(e)
                A = x @ c.abs()
                off = (D + 4) * 2.0 ** -24 * smax + 2.0 ** -23 * (1.45 * smax + e.abs().max() + 64)
                sums = 2 * (N / 16 + 32) * 2.0 ** -24
                seen = (~hidden).double() @ c.abs()
                f = torch.ones_like(la) if a == 0 else -la
                y = y + f * (x @ c)
                d = d + f.abs() * ((2.0 ** -11 + 2 * off + sums)[:, None] * A + 2.0 ** -32 * x.amax(1, keepdim=True) * seen)
                total = total + f.abs() * A
            d = d + 2.0 ** -22 * total
            out[at, heads], room[at, heads] = y.view(n, G, D), (d + u * (y.abs() + d) + z).view(n, G, D)
        first += n
    return out, room


def to_fp16(c, power):
    """c as fp16 holds it times 2^power: to nearest even, in steps of 2^-24 at least."""
    return (c * 2.0 ** power).to(torch.float16).double() * 2.0 ** -power
