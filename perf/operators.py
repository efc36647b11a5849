"""The operators of a serving node's window, as cases that can be timed and
compared: the tables of a paged cache, the cache's writes and reads, and the
attention over it.

A node keeps the keys and values of its running requests in pages of `page`
tokens.  A page's codes are 8 bits wide and carry one scale, a power of two, per
head and per side (keys, values).  One window's work is

    plan    block tables and slot maps from the requests' lengths
    append  the window's new keys and values into the pages
    attend  attention of the new tokens over everything cached
    export  cached tokens back as dense tensors
    step    plan, append and attend together, one layer of a window

and a case is a dict of plain values:

    kind             which of them ("append" also exports what it wrote)
    R                requests (rows of the block table)
    past_lo, past_hi tokens a request holds before the window (spread over their logarithm)
    add_lo, add_hi   new tokens of a request that brings a prompt or a chunk of one
    part             share of the requests that bring one; the others bring one token each
    ends             share of the requests that end in this window (kind "plan")
    spare            free pages of the pool over the pages that the window asks for
    page             tokens of a page
    heads, group     key and value heads, query heads that share one of them
    dim              numbers of a head
    form             "e4m3" or "int8", how the cache holds them
    dtype            "bf16" or "fp16" of queries, new keys and values, and outputs
    lse              1: attention also returns its log sums
    shape            the seed of the lengths: they belong to the case, the data to the pass

Lengths, codes and pages are as a running node has them: pages of a request
scattered over the pool, keys and values near normal with a magnitude of its own
for each page and head, queries and new keys and values views into one wide
projection's output.
"""
import math
import random

import torch

own = False

E_MIN = -64                                     # the smallest exponent of a page's scale
DTYPE = {"bf16": torch.bfloat16, "fp16": torch.float16}


def _case(name, kind, R, past, add=(1, 1), part=0.0, ends=0.0, spare=1.25, page=16, heads=8, group=4, dim=128,
          form="e4m3", dtype="bf16", lse=0, shape=1):
    return dict(name=name, kind=kind, R=R, past_lo=past[0], past_hi=past[1], add_lo=add[0], add_hi=add[1], part=part,
                ends=ends, spare=spare, page=page, heads=heads, group=group, dim=dim, form=form, dtype=dtype, lse=lse,
                shape=shape)


def listed():
    return [
        # one request's next token: a call is a launch's latency
        _case("plan_one", "plan", 1, (500, 500)),
        # a node's running and queued requests in a window of continuous batching: some bring prompts, some end
        _case("plan_window", "plan", 264, (1, 4096), (100, 4000), part=0.2, ends=0.1),
        # the tables of many nodes in one call, with a pool that runs short
        _case("plan_fleet", "plan", 16384, (1, 8192), (1, 1000), part=0.1, ends=0.05, spare=0.9),
        # the next token of every running request
        _case("append_tokens", "append", 64, (1, 8192), page=32, dim=64, form="int8", dtype="fp16"),
        # prompts of odd lengths, some continuing a page that holds tokens already
        _case("append_prompts", "append", 24, (1, 200), (100, 2000), part=1.0),
        # one request's next token after a short prompt: latency
        _case("attend_one", "attend", 1, (777, 777)),
        # the next token of every running request, lengths spread widely
        _case("attend_tokens", "attend", 64, (100, 8192), form="int8", dtype="fp16"),
        # long contexts, a cache past 4 GB: memory's rate
        _case("attend_long", "attend", 24, (60000, 131071), page=64, group=8, lse=1),
        # one head that all query heads share, a few tokens at once (drafted tokens that are checked)
        _case("attend_shared", "attend", 200, (1, 3000), (2, 4), part=0.7, page=64, heads=1, group=16, dim=64,
              form="int8"),
        # chunks of prompts beside single tokens, as a window of continuous batching has them
        _case("attend_mixed", "attend", 48, (1, 6000), (256, 1024), part=0.2, page=32, dtype="fp16"),
        # one long prompt: the matrix cores' rate
        _case("attend_prompt", "attend", 1, (1, 1), (16380, 16380), part=1.0, page=64),
        # one layer of a window of single tokens, tables and cache write included
        _case("step_tokens", "step", 64, (100, 2000), heads=4, group=8, dim=256),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["plan", "append", "attend", "attend", "attend", "step"])
    common = dict(page=rng.choice([16, 32, 64, 128]), form=rng.choice(["e4m3", "int8"]),
                  dtype=rng.choice(["bf16", "fp16"]), shape=rng.randrange(1, 1 << 20))
    if kind == "plan":
        R = _log(rng, 1, 16384)
        c = _case("", kind, R, (1, _log(rng, 20, 8192)), (1, _log(rng, 2, 4000 if R < 2000 else 1000)),
                  part=rng.choice([0.0, 0.1, 0.3]), ends=rng.choice([0.0, 0.05, 0.2]), spare=rng.choice([0.8, 1.0, 1.5]),
                  page=common["page"], shape=common["shape"])
        del c["name"]
        return c
    dim = rng.choice([64, 128, 256])
    heads = rng.choice([1, 2, 4, 8])
    group = rng.choice([1, 2, 3, 4, 5, 7, 8, 16]) if heads * dim <= 1024 else rng.choice([1, 3, 4, 8])
    shape = rng.choice(["tokens", "few", "mixed", "prompt"])
    wide = heads * dim                          # numbers of a token, keys alone
    if shape == "prompt":
        R = _log(rng, 1, 16)
        past, add, part = (1, _log(rng, 2, 2000)), None, 1.0
        hi = _log(rng, 40, max(50, min(12000 * 1024 // (wide * group), 16000 // R)))
        add = (max(1, hi // 3), hi)
    elif shape == "mixed":
        R = _log(rng, 8, 100)
        past, add, part = (1, _log(rng, 200, 6000)), (17, _log(rng, 40, 800)), 0.2
    else:
        R = _log(rng, 1, 256)
        hi = _log(rng, 30, max(100, min(131071, (1 << 30) // (R * wide))))
        past, add, part = (max(1, hi // 40), hi), (2, 5), 0.6 if shape == "few" else 0.0
    c = _case("", kind, R, past, add, part=part, heads=heads, group=group, dim=dim, lse=rng.choice([0, 1]), **common)
    del c["name"]
    return c


# ---- what a case's lengths are ------------------------------------------------------------------------------------

def _lengths(case):
    """past and add of every request, plain lists."""
    rng = random.Random(case["shape"])
    past = [_log(rng, case["past_lo"], case["past_hi"]) for _ in range(case["R"])]
    add = [1] * case["R"]
    n = int(math.ceil(case["part"] * case["R"]))
    for i in rng.sample(range(case["R"]), n):
        add[i] = _log(rng, case["add_lo"], case["add_hi"])
    for i in rng.sample(range(case["R"]), int(case["ends"] * case["R"])):
        add[i] = -1
    return past, add


def _sizes(case):
    """The table's width, the pool's pages, and the tokens that the window may bring."""
    past, add = _lengths(case)
    page = case["page"]
    held = sum(-(-p // page) for p in past)
    asked = sum(-(-(p + a) // page) - -(-p // page) for p, a in zip(past, add) if a > 0)
    width = max(-(-(p + max(a, 0)) // page) for p, a in zip(past, add)) + 3
    tokens = sum(a for a in add if a > 0)
    # a window's buffers are a little wider than its tokens
    return past, add, width, held + int(asked * case["spare"]) + (1 if case["spare"] >= 1 else 0), tokens, tokens + 3


def _randn(shape, gen):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)


def _pow2(e):
    return ((e + 127).clamp(1, 254) << 23).to(torch.int32).view(torch.float32)


def _need(amax, form):
    """The smallest exponent e with amax <= 448 * 2^e (e4m3) or 127 * 2^e (int8)."""
    f, x = torch.frexp(amax)
    if form == "e4m3":
        e = torch.where(f <= 0.875, x - 9, x - 8)
    else:
        e = torch.where(f <= 0.9921875, x - 7, x - 6)
    return torch.where(amax > 0, e.clamp(min=E_MIN), torch.full_like(e, E_MIN)).to(torch.int32)


def _encode(y, form):
    """Codes of y, already divided by its scale."""
    if form == "e4m3":
        return y.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    return y.round().clamp(-127, 127).to(torch.int8).view(torch.uint8)


def _decode(codes, form):
    return codes.view(torch.float8_e4m3fn if form == "e4m3" else torch.int8).float()


def _tables(case, gen):
    """Lengths, block table and ring of free pages, as a running node has them."""
    past, add, width, pages, tokens, limit = _sizes(case)
    R, page = case["R"], case["page"]
    order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    held = torch.tensor([-(-p // page) for p in past], dtype=torch.int64, device="cuda")
    base = torch.cumsum(held, 0) - held
    col = torch.arange(width, device="cuda")
    inside = col[None, :] < held[:, None]
    table = torch.zeros(R, width, dtype=torch.int32, device="cuda")
    table[inside] = order[(base[:, None] + col[None, :])[inside]]
    free = order[int(held.sum()):].contiguous()
    return dict(past=torch.tensor(past, dtype=torch.int32, device="cuda"),
                add=torch.tensor(add, dtype=torch.int32, device="cuda"), table=table, free=free, pages=pages,
                width=width, tokens=tokens, limit=limit)


def _inputs(case, seed):
    """Everything that the seed decides, the same for both sides."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = _tables(case, gen)
    if case["kind"] == "plan":
        return s
    H, G, D, page = case["heads"], case["group"], case["dim"], case["page"]
    codes = torch.empty(s["pages"], H, 2, page, D, dtype=torch.uint8, device="cuda")
    exps = torch.empty(s["pages"], H, 2, dtype=torch.int32, device="cuda")
    block = max(1, (1 << 27) // (H * 2 * page * D))
    for p in range(0, s["pages"], block):
        q = min(s["pages"], p + block)
        mag = torch.exp2(2 * torch.rand(q - p, H, 2, generator=gen, device="cuda") - 1)
        x = _randn((q - p, H, 2, page, D), gen) * mag[..., None, None]
        exps[p:q] = _need(x.abs().amax(dim=(3, 4)), case["form"])
        codes[p:q] = _encode(x * _pow2(-exps[p:q])[..., None, None], case["form"])
        del x
    s["codes"], s["exps"] = codes, exps
    # one projection's output, of which queries, keys and values are views
    wide = _randn((s["limit"], (H * G + 2 * H) * D), gen).to(DTYPE[case["dtype"]])
    s["q"] = wide[:, :H * G * D].unflatten(1, (H * G, D))
    s["k"] = wide[:, H * G * D:(H * G + H) * D].unflatten(1, (H, D))
    s["v"] = wide[:, (H * G + H) * D:].unflatten(1, (H, D))
    s["scale"] = 1.0 / math.sqrt(D)
    return s


def _wanted(case, s):
    """Slots of every cached token of the pages that the window writes to."""
    page = case["page"]
    plan = _plan(s, page)
    table = plan["table"].tolist()
    out = []
    for i, (p, g) in enumerate(zip(s["past"].tolist(), plan["granted"].tolist())):
        if g:
            out += [table[i][t // page] * page + t % page for t in range(p // page * page, p + g)]
    return torch.tensor(out, dtype=torch.int64, device="cuda")


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if case["kind"] == "append":
        s["wanted"] = _wanted(case, s)
    if own:
        from paper_2508_01744_amd import KvCache, KvTables, kv_config
        cfg = kv_config(case["R"], s["width"] * case["page"], s["pages"], page=case["page"], heads=case["heads"],
                        group=case["group"], dim=case["dim"], form=case["form"])
        s["tables"] = KvTables(cfg)
        s["tables"].load(s["past"], s["table"], s["free"])
        s["max_new"] = max(1, max(s["add"].tolist()))
        s["step"] = s["tables"].plan(s["add"], s["limit"], max_new=s["max_new"])
        if case["kind"] != "plan":
            s["cache"] = KvCache(cfg)
            s["cache"].load(s["codes"], s["exps"])
            del s["codes"], s["exps"]
            s["out"] = torch.empty(s["limit"], case["heads"] * case["group"], case["dim"],
                                   dtype=DTYPE[case["dtype"]], device="cuda")
            s["lse"] = torch.empty(s["limit"], case["heads"] * case["group"], device="cuda") if case["lse"] else None
    elif case["kind"] != "plan":
        s["plan"] = _plan(s, case["page"])
    return s


# ---- one pass -----------------------------------------------------------------------------------------------------

def run(state):
    kind = state["case"]["kind"]
    return (_run_own if own else _run_plain)(state, kind)


def _run_own(s, kind):
    if kind == "plan":
        return _plan_outputs(s["tables"].plan(s["add"], s["limit"], max_new=s["max_new"], step=s["step"]), s["tables"])
    if kind == "append":
        s["cache"].append(s["step"], s["k"], s["v"])
        return s["cache"].export(s["wanted"], s["k"].dtype)
    if kind == "step":
        s["tables"].plan(s["add"], s["limit"], max_new=s["max_new"], step=s["step"])
        s["cache"].append(s["step"], s["k"], s["v"])
    s["cache"].attend(s["tables"], s["step"], s["q"], out=s["out"], lse=s["lse"], scale=s["scale"])
    n = s["tokens"]
    result = (s["out"][:n], s["lse"][:n]) if s["lse"] is not None else (s["out"][:n],)
    return (s["step"].slots, *result) if kind == "step" else result


def _plan_outputs(step, tables):
    return dict(starts=step.starts, granted=step.granted, slots=step.slots, lengths=step.lengths,
                counters=step.counters, table=tables.table, ring=tables.ring)


def _run_plain(s, kind):
    case = s["case"]
    if kind == "plan":
        return _plan(s, case["page"])
    if kind == "append":
        _append(s, s["plan"], case)
        return _export(s, s["wanted"], case)
    plan = s["plan"]
    if kind == "step":
        plan = _plan(s, case["page"])
        _append(s, plan, case)
    result = _attend(s, plan, case)
    return (plan["slots"], *result) if kind == "step" else result


# ---- the plain forms ----------------------------------------------------------------------------------------------

def _plan(s, page):
    past, add, limit, pages = s["past"].long(), s["add"].long(), s["limit"], s["pages"]
    table = s["table"].clone()
    ring = torch.zeros(pages, dtype=torch.int32, device=past.device)
    n_free = s["free"].numel()
    ring[:n_free] = s["free"]
    held = (past + page - 1) // page
    ask = torch.where((add > 0) & (past + add <= s["width"] * page), add, torch.zeros_like(add))
    need = (past + ask + page - 1) // page - held
    cum, tok = torch.cumsum(need, 0), torch.cumsum(ask, 0)
    ok = (ask > 0) & ((need == 0) | (cum <= n_free)) & (tok <= limit)
    granted = torch.where(ok, ask, torch.zeros_like(ask))
    starts = torch.cat([torch.zeros_like(tok[:1]), tok]).clamp(max=limit)
    # slots: the request of every token, its position, its page
    t = torch.arange(limit, device=past.device)
    i = torch.searchsorted(tok, t, right=True)
    here = (t < tok[-1]) & ok[i.clamp(max=past.numel() - 1)]
    i = i.clamp(max=past.numel() - 1)
    pos = past[i] + t - starts[i]
    n = pos // page
    fresh = n >= held[i]
    taken_at = torch.where(here, cum[i] - need[i] + n - held[i], torch.zeros_like(n))
    old = table[i, torch.where(here & ~fresh, n, torch.zeros_like(n))].long()
    ids = torch.where(fresh, ring[taken_at.clamp(min=0) % pages].long(), old)
    slots = torch.where(here, ids * page + pos % page, torch.full_like(pos, -1))
    first = here & fresh & (pos % page == 0)
    table[i[first], n[first]] = ids[first].to(torch.int32)
    # pages of the requests that end go to the ring's tail, in the requests' order
    ended = add < 0
    gone = ended[:, None] & (torch.arange(s["width"], device=past.device)[None, :] < held[:, None])
    given = s["table"][gone]
    ring[(n_free + torch.arange(given.numel(), device=past.device)) % pages] = given
    taken = torch.where(ok, need, torch.zeros_like(need)).sum()
    zero = torch.zeros_like(taken)
    counters = torch.stack([taken % pages, n_free - taken + given.numel(), starts[-1],
                            ((add > 0) & ~ok).sum(), taken, zero + given.numel(), zero, zero])
    lengths = torch.where(ended, torch.zeros_like(past), past + granted)
    i32 = torch.int32
    return dict(starts=starts.to(i32), granted=granted.to(i32), slots=slots, lengths=lengths.to(i32),
                counters=counters.to(i32), table=table, ring=ring)


def _append(s, plan, case):
    form, page, H = case["form"], case["page"], case["heads"]
    codes, exps = s["codes"], s["exps"]
    slots = plan["slots"]
    live = slots >= 0
    slot = slots[live]
    ids, off = slot // page, slot % page
    x = torch.stack([s["k"][live].float(), s["v"][live].float()], 2)          # [n][H][2][D]
    amax = torch.zeros(s["pages"], H, 2, device=x.device)
    amax.scatter_reduce_(0, ids[:, None, None].expand(-1, H, 2), x.abs().amax(-1), "amax")
    need = _need(amax, form)
    touched = torch.unique(ids)
    fresh = torch.zeros(s["pages"], dtype=torch.bool, device=x.device)
    fresh[ids[off == 0]] = True
    before = exps[touched]
    after = torch.where(fresh[touched][:, None, None], need[touched], torch.maximum(before, need[touched]))
    kept = _decode(codes[touched], form) * _pow2(torch.clamp(before - after, max=0))[..., None, None]
    codes[touched] = _encode(kept, form)
    exps[touched] = after
    codes[ids, :, :, off] = _encode(x * _pow2(-exps[ids])[..., None], form)


def _export(s, slots, case):
    ids, off = slots // case["page"], slots % case["page"]
    x = _decode(s["codes"][ids, :, :, off], case["form"]) * _pow2(s["exps"][ids])[..., None]
    x = x.to(DTYPE[case["dtype"]])
    return x[:, :, 0].contiguous(), x[:, :, 1].contiguous()


def _attend(s, plan, case):
    H, G, D, page, form = case["heads"], case["group"], case["dim"], case["page"], case["form"]
    n_all = s["tokens"]
    out = torch.zeros(n_all, H * G, D, device="cuda")
    lse = torch.full((n_all, H * G), float("-inf"), device="cuda")
    past, granted, starts = _host(s, plan)
    for i in range(case["R"]):
        n = granted[i]
        if n <= 0:
            continue
        L = past[i] + n
        ids = plan["table"][i, :-(-L // page)].long()
        kv = _decode(s["codes"][ids], form) * _pow2(s["exps"][ids])[..., None, None]   # [pages][H][2][page][D]
        kt = kv[:, :, 0].permute(1, 3, 0, 2).reshape(H, D, -1)[:, :, :L].contiguous()
        v = kv[:, :, 1].permute(1, 0, 2, 3).reshape(H, -1, D)[:, :L].contiguous()
        rows = max(1, min(n, (1 << 29) // (H * G * L)))
        for a in range(0, n, rows):
            b = min(n, a + rows)
            q = s["q"][starts[i] + a:starts[i] + b].float().unflatten(1, (H, G)).permute(1, 0, 2, 3).reshape(H, -1, D)
            sc = torch.bmm(q, kt) * s["scale"]                                        # [H][rows * G][L]
            if n > 1:
                last = past[i] + torch.arange(a, b, device="cuda").repeat_interleave(G)
                sc = sc.masked_fill(torch.arange(L, device="cuda")[None, :] > last[:, None], float("-inf"))
            m = sc.amax(-1, keepdim=True)
            p = torch.exp(sc - m)
            l = p.sum(-1, keepdim=True)
            o = torch.bmm(p, v) / l
            at = slice(starts[i] + a, starts[i] + b)
            out[at] = o.unflatten(1, (b - a, G)).permute(1, 0, 2, 3).reshape(b - a, H * G, D)
            lse[at] = (m + torch.log(l))[..., 0].unflatten(1, (b - a, G)).permute(1, 0, 2).reshape(b - a, H * G)
    out = out.to(DTYPE[case["dtype"]])
    return (out, lse) if case["lse"] else (out,)


def _host(s, plan):
    """The lengths as the program knows them on the host already (made from the requests, not copied back)."""
    past, add, width, pages, tokens, limit = _sizes(s["case"])
    granted, starts, at = [], [], 0
    for a in add:
        granted.append(max(a, 0))
        starts.append(at)
        at += max(a, 0)
    return past, granted, starts


# ---- what a pass cannot do without --------------------------------------------------------------------------------

def work(case):
    past, add, width, pages, tokens, limit = _sizes(case)
    H, G, D, page = case["heads"], case["group"], case["dim"], case["page"]
    wide = H * D
    asked = sum(-(-(p + a) // page) - -(-p // page) for p, a in zip(past, add) if a > 0)
    plan_bytes = 5 * 4 * case["R"] + 8 * limit + 8 * asked + 8 * sum(-(-p // page) for p, a in zip(past, add) if a < 0)
    plan_ops = 10 * case["R"] + 4 * limit
    if case["kind"] == "plan":
        return {"bytes": plan_bytes, "flops": plan_ops}
    append_bytes = tokens * wide * 2 * (2 + 1)
    if case["kind"] == "append":
        n = sum(p + a - p // page * page for p, a in zip(past, add))
        return {"bytes": append_bytes + n * wide * 2 * (1 + 2), "flops": tokens * wide * 2 * 3 + n * wide * 2}
    keys = sum(a * p + a * (a + 1) // 2 for p, a in zip(past, add))
    held = sum(p + a for p, a in zip(past, add))
    attend_bytes = held * wide * 2 + -(-held // page) * H * 8 + 2 * tokens * wide * G * 2
    flops = 4 * D * H * G * keys
    if case["kind"] == "step":
        return {"bytes": plan_bytes + append_bytes + attend_bytes, "flops": flops}
    return {"bytes": attend_bytes, "flops": flops}


# ---- the definition, in 64 bits -----------------------------------------------------------------------------------

_E4M3 = [(-1.0 if c & 128 else 1.0) * (float("nan") if c & 127 == 127 else
         math.ldexp(c & 7, -9) if (c >> 3) & 15 == 0 else math.ldexp(8 + (c & 7), ((c >> 3) & 15) - 10))
         for c in range(256)]


def _values64(codes, form):
    table = _E4M3 if form == "e4m3" else [c if c < 128 else c - 256 for c in range(256)]
    return torch.tensor(table, dtype=torch.float64, device=codes.device)[codes.long()]


def _round64(y, form):
    """y to the nearest value that a code stands for, ties to the even one (|y| within the range)."""
    if form == "int8":
        return torch.round(y)
    _, x = torch.frexp(y)
    quantum = torch.exp2((x - 1).clamp(min=-6).double() - 3)
    return torch.round(y / quantum) * quantum


def _exponent64(top, form):
    """The smallest e >= E_MIN whose range holds the number top."""
    e, most = E_MIN, 448.0 if form == "e4m3" else 127.0
    if top > most * 2.0 ** E_MIN:
        e = math.ceil(math.log2(top / most)) - 1
        while top > most * 2.0 ** e:
            e += 1
    return e


def _exact_plan(case, s):
    past, add, width, pages, tokens, limit = _sizes(case)
    page, free = case["page"], s["free"].tolist()
    ring = free + [0] * (pages - len(free))
    table = s["table"].tolist()
    old = [list(row) for row in table] if case["ends"] else table
    starts, granted, lengths, slots, back = [0], [], [], [-1] * limit, []
    at = cum = taken = refused = 0
    for i, (p, a) in enumerate(zip(past, add)):
        have = -(-p // page)
        if a < 0:
            back += old[i][:have]
        ask = a if 0 < a <= width * page - p else 0
        need = -(-(p + ask) // page) - have
        first = cum
        cum += need
        ok = ask > 0 and (need == 0 or cum <= len(free)) and at + ask <= limit
        if ok:
            taken += need
            for n in range(need):
                table[i][have + n] = ring[(first + n) % pages]
            for t in range(p, p + ask):
                slots[at + t - p] = table[i][t // page] * page + t % page
        refused += a > 0 and not ok
        granted.append(ask if ok else 0)
        lengths.append(0 if a < 0 else p + granted[-1])
        at += ask
        starts.append(min(at, limit))
    for n, g in enumerate(back):
        ring[(len(free) + n) % pages] = g
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")                     # noqa: E731
    counters = [taken % pages, len(free) - taken + len(back), starts[-1], refused, taken, len(back), 0, 0]
    return dict(starts=i32(starts), granted=i32(granted), slots=torch.tensor(slots, device="cuda"),
                lengths=i32(lengths), counters=i32(counters), table=i32(table), ring=i32(ring))


def _exact_pages(case, s, plan):
    """Values of the pages that the window writes to, after it: {page: [H][2][page][D]} in 64 bits, with exponents."""
    page, form, H = case["page"], case["form"], case["heads"]
    slots = plan["slots"].tolist()
    runs = {}
    for t, slot in enumerate(slots):
        if slot >= 0:
            runs.setdefault(slot // page, []).append((slot % page, t))
    ids = list(runs)
    at = {p: n for n, p in enumerate(ids)}
    index = torch.tensor(ids, device="cuda")
    old = s["exps"][index].double()
    values = _values64(s["codes"][index], form)
    x = torch.stack([s["k"].double(), s["v"].double()], 2)
    owner = torch.tensor([at[z // page] if z >= 0 else len(ids) for z in slots], device="cuda")
    top = torch.zeros(len(ids) + 1, H, 2, dtype=torch.float64, device="cuda")
    top.scatter_reduce_(0, owner[:, None, None].expand(-1, H, 2), x.abs().amax(-1), "amax")
    need = torch.tensor([_exponent64(z, form) for z in top[:-1].flatten().tolist()], dtype=torch.float64,
                        device="cuda").view(-1, H, 2)
    fresh = torch.tensor([runs[p][0][0] == 0 for p in ids], device="cuda")[:, None, None]
    new = torch.where(fresh, need, torch.maximum(old, need))
    values = _round64(values * torch.exp2(torch.clamp(old - new, max=0))[..., None, None], form)
    live = [t for t, z in enumerate(slots) if z >= 0]
    own_page = owner[live]
    values[own_page, :, :, torch.tensor([slots[t] % page for t in live], device="cuda")] = _round64(
        x[live] * torch.exp2(-new[own_page])[..., None], form)
    return at, values * torch.exp2(new)[..., None, None]


def exact(case, seed):
    s = _inputs(case, seed)
    if case["kind"] == "plan":
        return _exact_plan(case, s)
    H, G, D, page, form = case["heads"], case["group"], case["dim"], case["page"], case["form"]
    plan = _exact_plan(case, s)
    at, written = ({}, None) if case["kind"] == "attend" else _exact_pages(case, s, plan)
    if case["kind"] == "append":
        slots = _wanted(case, s).tolist()
        got = written[torch.tensor([at[z // page] for z in slots], device="cuda"), :, :,
                      torch.tensor([z % page for z in slots], device="cuda")]
        return got[:, :, 0].contiguous(), got[:, :, 1].contiguous()
    past, add, width, pages, tokens, limit = _sizes(case)
    table = plan["table"].tolist()
    out = torch.zeros(tokens, H * G, D, dtype=torch.float64, device="cuda")
    lse = torch.full((tokens, H * G), float("-inf"), dtype=torch.float64, device="cuda")
    first = 0
    for i, (p, n) in enumerate(zip(past, plan["granted"].tolist())):
        if n:
            ids = torch.tensor(table[i][:-(-(p + n) // page)], device="cuda")
            for h in range(H):
                kv = _values64(s["codes"][ids, h], form) * torch.exp2(s["exps"][ids, h].double())[..., None, None]
                for m, g in enumerate(table[i][:ids.numel()] if at else ()):
                    if g in at:
                        kv[m] = written[at[g], h]
                k = kv[:, 0].reshape(-1, D)[:p + n]
                v = kv[:, 1].reshape(-1, D)[:p + n].contiguous()
                kt = k.t().contiguous()
                for a in range(0, n, 1024):
                    b = min(n, a + 1024)
                    q = s["q"][first + a:first + b, h * G:(h + 1) * G].double()
                    for g in range(G):
                        sc = q[:, g].contiguous() @ kt * s["scale"]
                        later = torch.arange(p + n, device="cuda")[None, :] > torch.arange(p + a, p + b, device="cuda")[:, None]
                        sc[later] = float("-inf")
                        both = torch.logsumexp(sc, -1)
                        out[first + a:first + b, h * G + g] = torch.exp(sc - both[:, None]) @ v
                        lse[first + a:first + b, h * G + g] = both
        first += max(add[i], 0)
    result = (out, lse) if case["lse"] else (out,)
    return (plan["slots"], *result) if case["kind"] == "step" else result
