"""Differential attention over a paged cache whose codes are given (kv_flat.Window),
in 64 bits, and how far from it a right kernel may be.

The bound.  Each map's sums y_a = sum_j w_j v_j, A_a = sum_j w_j |v_j|, are off by
kv_flat's bound without the output's own rounding:

    D_a = 2^-11 A_a + (2 e + sums) A_a + N 2^-32 max(w_j 2^e_j) cmax

with e_j the larger of a page's two value exponents (the probabilities carry it).
Where the other head's exponent lies d below, its codes reach fp16 times 2^(lift -
d) (lift 7, e4m3; 5, int8): exact while that is at least fp16's smallest step over
the code's own, 2^-24 / 2^-9 or 2^-24, so for d <= 22 or 29; beyond, each code is
off by up to 2^-25 before 2^(d - lift) brings it back, so by 2^(d - lift - 25).
The difference y = y_0 - lambda y_1 and its factors are fp32:

    D = D_0 + |lambda| D_1 + 2^-22 (A_0 + |lambda| A_1)

Without a weight out is off by |gain| D + u |out| + z (u, z: kv_flat).  With one,
r = 1 / sqrt(mean(y^2) + eps): mean((y + d)^2) + eps = (1 + x) / r^2 with |x| <= E =
r^2 (2 mean(|y| D) + mean(D^2)), and is eps at least.  So the kernel's r' is at least
r (1 + E)^-1/2 and at most R = r (1 - E)^-1/2 (E < 1) and eps^-1/2, and with

    |y' r' - y r| <= |y' - y| r' + |y| |r' - r|

out is off by |gain weight| (D R + |y| max(R - r, r - r (1 + E)^-1/2)), by 2^-21 of
|gain weight y r| for the sum, root and division in fp32, and by u |out| + z.  (Where
the maps nearly cancel E passes 1: a row of one key whose lambda is near 1.)"""
import math

import torch

from kv_flat import E4M3, INT8

LIFT = {"e4m3": 7, "int8": 5}
STEP = {"e4m3": -9, "int8": 0}      # the codes' own smallest step, as a power of two


def lambdas(window, per_token, seed=0):
    gen = torch.Generator(device=window.device).manual_seed(seed)
    ho = window.heads // 2 * window.group
    shape = (window.tokens, ho) if per_token else (ho,)
    return torch.rand(shape, generator=gen, device=window.device) * 1.2 - 0.1


def weights(window, seed=0):
    gen = torch.Generator(device=window.device).manual_seed(seed + 1)
    return 1 + 0.3 * torch.randn(2 * window.dim, generator=gen, device=window.device)


def reference(w, lam, weight, gain, eps, spoil=None):
    """out, lse, and the bounds on both.  spoil(y [pairs' rows][2 dim]): a mistake planted in the difference."""
    values = torch.tensor(E4M3 if w.form == "e4m3" else INT8, dtype=torch.float64, device=w.device)
    G, D = w.group, w.dim
    pairs = w.heads // 2
    lam = lam.double().expand(w.tokens, pairs * G)
    out = torch.zeros(w.tokens, pairs * G, 2 * D, dtype=torch.float64, device=w.device)
    room = torch.zeros_like(out)
    lse = torch.zeros(w.tokens, w.heads * G, dtype=torch.float64, device=w.device)
    lse_room = torch.zeros_like(lse)
    u, z = (2.0 ** -8, 0.0) if w.dtype == torch.bfloat16 else (2.0 ** -11, 2.0 ** -25)
    first = 0
    for past, n, row in zip(w.past, w.add, w.rows):
        if n <= 0:
            continue
        N = past + n
        ids = torch.tensor(row, device=w.device)
        last = past + torch.arange(n, device=w.device).repeat_interleave(G)
        hidden = torch.arange(N, device=w.device)[None, :] > last[:, None]
        at = slice(first, first + n)
        for p in range(pairs):
            code = values[w.codes[ids, 2 * p:2 * p + 2].long()]                        # [pages][2][2][page][D]
            e = w.exps[ids, 2 * p:2 * p + 2].double()
            kv = code * torch.exp2(e)[..., None, None]
            v = torch.cat([kv[:, a, 1].reshape(-1, D)[:N] for a in (0, 1)], 1)
            top = e[:, :, 1].amax(1)
            fall = top[:, None] - e[:, :, 1] - LIFT[w.form]                            # codes reach fp16 times 2^-fall
            lossy = STEP[w.form] - fall < -24
            loss = torch.where(lossy, torch.exp2(fall + e[:, :, 1] - 25), torch.zeros_like(fall))
            loss = loss[:, :, None, None].expand(-1, -1, w.page, D)
            loss = torch.cat([loss[:, a].reshape(-1, D)[:N] for a in (0, 1)], 1)
            ev = top.repeat_interleave(w.page)[:N]
            y, d, total = 0.0, 0.0, 0.0
            la = lam[at, p * G:(p + 1) * G].reshape(-1, 1)
            for a in (0, 1):
                k = kv[:, a, 0].reshape(-1, D)[:N].contiguous()
                heads = slice((2 * p + a) * G, (2 * p + a + 1) * G)
                q = w.q[at, heads].double().reshape(n * G, D)
                s = (q @ k.t().contiguous()) * w.scale
                s.masked_fill_(hidden, -math.inf)
                smax = ((q.abs() @ k.abs().t().contiguous()) * w.scale).masked_fill_(hidden, 0).amax(1)
                x = torch.softmax(s, 1)
                both = torch.logsumexp(s, 1)
                A = x @ v.abs()
                off = (D + 4) * 2.0 ** -24 * smax + 2.0 ** -23 * (1.45 * smax + ev.abs().max() + 64)
                sums = 2 * (N / 16 + 32) * 2.0 ** -24
                gone = N * 2.0 ** -32 * (x * torch.exp2(ev)).amax(1) * code[:, :, 1].abs().max()
                f = torch.ones_like(la) if a == 0 else -la
                y = y + f * (x @ v)
                d = d + f.abs() * ((2.0 ** -11 + 2 * off + sums)[:, None] * A + gone[:, None] + x @ loss)
                total = total + f.abs() * A
                lse[at, heads] = both.view(n, G)
                lse_room[at, heads] = (off + sums + 2.0 ** -22 * (1 + both.abs())).view(n, G)
            d = d + 2.0 ** -22 * total
            if spoil is not None:
                y = spoil(y)
            if weight is None:
                o, tol = gain * y, abs(gain) * d
            else:
                r = 1 / torch.sqrt(y.square().mean(1, keepdim=True) + eps)
                E = r * r * (2 * (y.abs() * d).mean(1, keepdim=True) + d.square().mean(1, keepdim=True))
                R = torch.where(E < 1, r / torch.sqrt((1 - E).clamp(min=1e-300)), math.inf).clamp(max=eps ** -0.5)
                by = gain * weight.double()
                o = by * r * y
                away = torch.maximum(R - r, r - r / torch.sqrt(1 + E))
                tol = by.abs() * (d * R + y.abs() * (away + 2.0 ** -21 * r))
            tol = tol + u * (o.abs() + tol) + z + 2.0 ** -40
            ho = slice(p * G, (p + 1) * G)
            out[at, ho], room[at, ho] = o.view(n, G, 2 * D), tol.view(n, G, 2 * D)
        first += n
    return out, lse, room, lse_room


def compare(w, per_token=False, norm=True, gain=0.3, eps=1e-5, max_new=None, tell="", on_gpu=None):
    """The kernels on this window against the reference."""
    tables, cache, step = on_gpu or w.on_gpu(max_new)
    lam, weight = lambdas(w, per_token), weights(w) if norm else None
    lse = torch.full((w.tokens, w.heads * w.group), 7.0, device=w.device)
    out = cache.attend_diff(tables, step, w.q, lam, weight=weight, gain=gain, eps=eps, lse=lse, scale=w.scale)
    ref, ref_lse, room, lse_room = reference(w, lam, weight, gain, eps)
    share, lse_share = (out.double() - ref).abs() / room, (lse.double() - ref_lse).abs() / lse_room
    print("  ", tell, "worst share of the bound", float(share.max()), "of the logarithm's", float(lse_share.max()), flush=True)
    assert bool((share <= 1).all()), (tell, float(share.max()), torch.nonzero(~(share <= 1))[:4].tolist())
    assert bool((lse_share <= 1).all()), (tell, float(lse_share.max()), torch.nonzero(~(lse_share <= 1))[:4].tolist())
    return tables, cache, step, out
