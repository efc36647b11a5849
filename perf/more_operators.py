"""More operators of a serving node's paged cache, as cases that can be timed and
compared: changes of which pages the requests hold, and differential attention.

A request's prompt is often continued more than once (samples, beams, an agent's
branches), continued tokens are taken back (drafts that were not accepted), and a
pool that has run for a while has free pages everywhere.  And models with
differential attention take the difference of two softmax maps over the same
values.

    fork     requests continue others' tokens: whole pages are shared, a partly filled last one is copied
    trim     requests keep their first tokens; pages that nobody holds any more go back
    compact  held pages move to the pool's lower end
    diff     (softmax(s q1 K1^T) - lambda softmax(s q2 K2^T)) [V1 V2] over the cached tokens
    sample   together: prompts forked, one token for each fork written and attended, forks ended

"fork" and "compact" copy the pages of one layer too, and return what the copies
hold.  A case is a dict of plain values:

    kind             which of them
    R                requests that hold tokens (with kids: families)
    past_lo, past_hi tokens that they hold (spread over their logarithm)
    kids             forks of each ("trim": requests that continue each one's prefix)
    add_lo, add_hi   new tokens of a request that brings a prompt or a chunk of one ("trim": tokens that a
                     kid holds behind what it shares)
    part             share of the requests that bring one; the others bring one token each ("fork": share
                     of the forks that take only the first part of the tokens)
    ends             share of the families and kids that end ("trim"), of the forks that cannot be made ("fork")
    back             share of the kids that take their last tokens back ("trim")
    spare            the pool's pages over those held ("fork": free pages over those that are asked for)
    page             tokens of a page
    heads, group     key and value heads, query heads that share one of them; heads 2 p and 2 p + 1 are a pair
    dim              numbers of a head
    form             "e4m3" or "int8", how the cache holds them
    dtype            "bf16" or "fp16" of queries, new keys and values, and outputs
    lam              "head" or "token": a lambda for each head, or for each token and head
    norm             1: each head's output is normalised and scaled
    lse              1: the log sums of both maps are returned too
    shape            the seed of the lengths: they belong to the case, the data to the pass

Pages of a request lie scattered over the pool, keys and values are near normal
with a magnitude of their own for each page and head, queries and new keys and
values are views into one wide projection's output.
"""
import math
import random

import torch

own = False

E_MIN = -64                                     # the smallest exponent of a page's scale
GAIN, EPS = 0.2, 1e-5                           # a layer's 1 - lambda_init, and of the norm
DTYPE = {"bf16": torch.bfloat16, "fp16": torch.float16}


def _case(name, kind, R, past, kids=0, add=(1, 1), part=0.0, ends=0.0, back=0.0, spare=1.25, page=16, heads=8, group=4,
          dim=128, form="e4m3", dtype="bf16", lam="head", norm=1, lse=0, shape=1):
    return dict(name=name, kind=kind, R=R, past_lo=past[0], past_hi=past[1], kids=kids, add_lo=add[0], add_hi=add[1],
                part=part, ends=ends, back=back, spare=spare, page=page, heads=heads, group=group, dim=dim, form=form,
                dtype=dtype, lam=lam, norm=norm, lse=lse, shape=shape)


def listed():
    return [
        # one request's second sample: a call is a launch's latency
        _case("fork_one", "fork", 1, (777, 777), kids=1),
        # four samples of every prompt of a node, some of a part of it, some that cannot be made
        _case("fork_samples", "fork", 66, (100, 8192), kids=4, part=0.1, ends=0.05, heads=4, dim=64, form="int8",
              dtype="fp16"),
        # the end of a window: samples that end, families that end whole, drafts taken back
        _case("trim_window", "trim", 52, (100, 4096), kids=4, add=(1, 600), ends=0.1, back=0.3),
        # the tables of many nodes in one call
        _case("trim_fleet", "trim", 5461, (1, 4096), kids=2, add=(1, 300), ends=0.05, back=0.2, page=32),
        # a node's pool with holes everywhere, one layer moved
        _case("compact_node", "compact", 64, (100, 4096), spare=1.4),
        # a pool of gigabytes: memory's rate
        _case("compact_large", "compact", 311, (1000, 40000), spare=1.3, page=64, form="int8", dtype="fp16"),
        # three samples of each prompt, their next token, and their end
        _case("sample_tokens", "sample", 21, (100, 2000), kids=3, page=32, dim=64),
        # one request's next token after a short prompt: latency
        _case("diff_one", "diff", 1, (777, 777)),
        # the next token of every running request, lengths spread widely
        _case("diff_tokens", "diff", 64, (100, 8192), form="int8", dtype="fp16", lam="token", lse=1),
        # long contexts, a cache past 4 GB: memory's rate
        _case("diff_long", "diff", 24, (60000, 131071), page=64, group=8),
        # chunks of prompts beside single tokens, as a window of continuous batching has them
        _case("diff_mixed", "diff", 48, (1, 6000), add=(256, 1024), part=0.2, page=32, heads=16, group=2, dim=64,
              norm=0),
        # one long prompt: the matrix cores' rate
        _case("diff_prompt", "diff", 1, (1, 1), add=(10001, 10001), part=1.0, page=128, form="int8"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["fork", "trim", "compact", "diff", "diff", "diff", "sample"])
    common = dict(page=rng.choice([16, 32, 64, 128]), form=rng.choice(["e4m3", "int8"]),
                  dtype=rng.choice(["bf16", "fp16"]), shape=rng.randrange(1, 1 << 20))
    heads, dim = rng.choice([2, 4, 8, 16]), rng.choice([64, 128])
    if kind == "fork":
        kids = rng.randrange(1, 6)
        R = _log(rng, 1, 600)
        c = _case("", kind, R, (1, _log(rng, 20, 8192)), kids=kids, part=rng.choice([0.0, 0.2, 0.5]),
                  ends=rng.choice([0.0, 0.1]), spare=rng.choice([0.8, 1.0, 1.5]), heads=min(heads, 8), dim=dim, **common)
    elif kind == "trim":
        kids = rng.randrange(0, 5)
        c = _case("", kind, _log(rng, 1, 12000 // (1 + kids)), (1, _log(rng, 20, 6000)), kids=kids,
                  add=(1, _log(rng, 2, 500)), ends=rng.choice([0.0, 0.05, 0.3]), back=rng.choice([0.0, 0.3, 1.0]),
                  **common)
    elif kind == "compact":
        R = _log(rng, 1, 300)
        hi = _log(rng, 20, max(40, min(100000, (1 << 29) // (R * heads * dim))))
        c = _case("", kind, R, (max(1, hi // 40), hi), spare=rng.choice([1.0, 1.1, 1.5, 2.5]), heads=heads, dim=dim,
                  **common)
    else:
        group = rng.choice([1, 2, 3, 4, 5, 7, 8]) if heads * dim <= 1024 else rng.choice([1, 3, 4])
        wide = heads * dim
        some = dict(heads=heads, group=group, dim=dim, lam=rng.choice(["head", "token"]), norm=rng.choice([0, 1]),
                    lse=rng.choice([0, 1]), **common)
        shape = rng.choice(["tokens", "few", "mixed", "prompt"])
        if kind == "sample":
            R, kids = _log(rng, 1, 40), rng.randrange(1, 6)
            c = _case("", kind, R, (1, _log(rng, 20, max(40, min(20000, (1 << 28) // (R * kids * wide))))), kids=kids,
                      **some)
        elif shape == "prompt":
            R = _log(rng, 1, 16)
            hi = _log(rng, 40, max(50, min(8000 * 1024 // (wide * group), 12000 // R)))
            c = _case("", kind, R, (1, _log(rng, 2, 2000)), add=(max(1, hi // 3), hi), part=1.0, **some)
        elif shape == "mixed":
            c = _case("", kind, _log(rng, 8, 100), (1, _log(rng, 200, 6000)), add=(17, _log(rng, 40, 600)), part=0.2,
                      **some)
        else:
            R = _log(rng, 1, 256)
            hi = _log(rng, 30, max(100, min(131071, (1 << 30) // (R * wide))))
            c = _case("", kind, R, (max(1, hi // 40), hi), add=(2, 5), part=0.6 if shape == "few" else 0.0, **some)
    del c["name"]
    return c


# ---- what a case's lengths are ------------------------------------------------------------------------------------

def _pages(n, page):
    return -(-n // page)


def _plan_of(case):
    """The case's requests on the host, plain lists: past (tokens held), start (pages shared with the family's first
    request), parent, and what is asked for, by kind: add; src, dst and tokens; keep."""
    rng = random.Random(case["shape"])
    R, kids, page = case["R"], case["kids"], case["page"]
    first = [_log(rng, case["past_lo"], case["past_hi"]) for _ in range(R)]
    rows = R * (1 + kids)
    o = dict(past=first + [0] * (rows - R), start=[0] * rows, parent=[i % R for i in range(rows)])
    if case["kind"] in ("fork", "sample"):
        dst = list(range(R, rows))
        rng.shuffle(dst)
        o["dst"], o["src"] = dst, [i % R for i in dst]
        o["tokens"] = [first[i] for i in o["src"]]
        for j in rng.sample(range(len(dst)), int(case["part"] * len(dst))):
            o["tokens"][j] = rng.randrange(0, o["tokens"][j] + 1)
        for j in rng.sample(range(len(dst)), int(case["ends"] * len(dst))):
            # of a request that holds nothing, onto one that holds something, or onto one that another fork takes
            o["src" if j % 3 == 0 else "dst"][j] = (dst[0], o["src"][j], dst[j - 1])[j % 3]
    if case["kind"] == "trim":
        keep = [-1] * rows
        for i in range(R, rows):
            shared = rng.randrange(0, first[i % R] + 1)
            o["start"][i] = shared // page
            o["past"][i] = shared + _log(rng, case["add_lo"], case["add_hi"])
        for i in rng.sample(range(R), int(math.ceil(case["ends"] * R))):
            for j in range(i, rows, R):
                keep[j] = 0
        for i in rng.sample(range(rows), int(case["ends"] * rows)):
            keep[i] = 0
        for i in range(rows):
            if keep[i] < 0 and rng.random() < case["back"]:
                keep[i] = max(0, o["past"][i] - rng.randrange(1, 9))
        o["keep"] = keep
    if case["kind"] == "sample":
        o["add"] = [0] * R + [1] * (rows - R)
        o["keep"] = [-1] * R + [0] * (rows - R)
    if case["kind"] == "diff":
        o["add"] = [1] * R
        for i in rng.sample(range(R), int(math.ceil(case["part"] * R))):
            o["add"][i] = _log(rng, case["add_lo"], case["add_hi"])
    return o


def _sizes(case):
    """The plan, the table's width, pages held and of the pool, and the window's tokens."""
    o, page = _plan_of(case), case["page"]
    held = sum(_pages(p, page) - s for p, s in zip(o["past"], o["start"]))
    width = max(_pages(p, page) for p in o["past"]) + 3
    tokens = 0
    pool = int(math.ceil(held * case["spare"])) + 1
    if case["kind"] == "fork":
        pool = held + int(sum(t % page > 0 for t in o["tokens"]) * case["spare"])
    if case["kind"] == "sample":
        tokens = sum(o["add"])
        pool = held + 2 * tokens + 1
    if case["kind"] == "diff":
        tokens = sum(o["add"])
        width = max(_pages(p + a, page) for p, a in zip(o["past"], o["add"])) + 3
        pool = sum(_pages(p + a, page) for p, a in zip(o["past"], o["add"])) + 2
    return o, width, held, max(pool, 1), tokens


def _moves(held, pool):
    """Held pages that lie where the free ones are to be."""
    return max(1, held * (pool - held) // pool)


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


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _inputs(case, seed):
    """Everything that the seed decides, the same for both sides."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    o, width, held, pool, tokens = _sizes(case)
    page, kind, rows = case["page"], case["kind"], len(o["past"])
    order = torch.randperm(pool, generator=gen, device="cuda")
    if kind == "compact":
        # as many free pages below the held ones' number as chance gives, the same for every seed
        up = _moves(held, pool)
        low, high = order[order < held], order[order >= held]
        order = torch.cat([x[torch.randperm(x.numel(), generator=gen, device="cuda")] for x in (
            torch.cat([low[up:], high[:up]]), torch.cat([low[:up], high[up:]]))])
    order = order.to(torch.int32)
    past, start, parent = (torch.tensor(o[k], device="cuda") for k in ("past", "start", "parent"))
    to = (past + page - 1) // page
    base = torch.cumsum(to - start, 0) - (to - start)
    col = torch.arange(width, device="cuda")[None, :]
    mine = (col >= start[:, None]) & (col < to[:, None])
    table = torch.zeros(rows, width, dtype=torch.int32, device="cuda")
    table[mine] = order[(base[:, None] + col - start[:, None])[mine]]
    table = torch.where(col < start[:, None], table[parent], table).contiguous()
    free = order[held:].contiguous()
    if kind == "diff":
        # the new tokens' pages come from the free ones, in the requests' order
        end = (past + torch.tensor(o["add"], device="cuda") + page - 1) // page
        base = torch.cumsum(end - to, 0) - (end - to)
        new = (col >= to[:, None]) & (col < end[:, None])
        table[new] = free[(base[:, None] + col - to[:, None])[new]]
    s = dict(case=case, rows=rows, width=width, pool=pool, tokens=tokens, limit=tokens + 3,
             past=_i32(o["past"]), table=table, free=free)
    s.update((k, _i32(o[k])) for k in ("src", "dst", "tokens", "keep", "add") if k in o and k != "tokens")
    if "tokens" in o:
        s["first"] = _i32(o["tokens"])
    if kind == "trim":
        return s
    H, G, D = case["heads"], case["group"], case["dim"]
    codes = torch.empty(pool, H, 2, page, D, dtype=torch.uint8, device="cuda")
    exps = torch.empty(pool, H, 2, dtype=torch.int32, device="cuda")
    block = max(1, (1 << 27) // (H * 2 * page * D))
    for p in range(0, pool, block):
        q = min(pool, p + block)
        mag = torch.exp2(2 * torch.rand(q - p, H, 2, generator=gen, device="cuda") - 1)
        x = _randn((q - p, H, 2, page, D), gen) * mag[..., None, None]
        exps[p:q] = _need(x.abs().amax(dim=(3, 4)), case["form"])
        codes[p:q] = _encode(x * _pow2(-exps[p:q])[..., None, None], case["form"])
        del x
    s["codes"], s["exps"] = codes, exps
    if kind in ("diff", "sample"):
        # one projection's output, of which queries, keys and values are views
        wide = _randn((s["limit"], (H * G + 2 * H) * D), gen).to(DTYPE[case["dtype"]])
        s["q"] = wide[:, :H * G * D].unflatten(1, (H * G, D))
        s["k"] = wide[:, H * G * D:(H * G + H) * D].unflatten(1, (H, D))
        s["v"] = wide[:, (H * G + H) * D:].unflatten(1, (H, D))
        s["scale"] = 1.0 / math.sqrt(D)
        # lambda as a layer's learned vectors or its projection give it
        rows_of = (s["limit"],) if case["lam"] == "token" else ()
        s["lam"] = torch.sigmoid(_randn((*rows_of, H // 2 * G), gen))
        s["weight"] = 1 + 0.1 * _randn((2 * D,), gen) if case["norm"] else None
    return s


def _wanted(case, s):
    """Slots of all tokens of the pages that the copies go to."""
    moves = (_fork(s, case["page"]) if case["kind"] == "fork" else _compact(s))["moves"][:, 1].long()
    moves = moves[moves >= 0]
    return (moves[:, None] * case["page"] + torch.arange(case["page"], device="cuda")).flatten()


def prepare(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if kind in ("fork", "compact"):
        s["wanted"] = _wanted(case, s)
    if own:
        from paper_2508_01744_amd import KvCache, KvTables, kv_config
        cfg = kv_config(s["rows"], s["width"] * case["page"], s["pool"], page=case["page"], heads=case["heads"],
                        group=case["group"], dim=case["dim"], form=case["form"])
        t = s["tables"] = KvTables(cfg)
        t.load(s["past"], s["table"], s["free"], shared=kind == "trim")
        if kind in ("fork", "sample"):
            s["edit"] = t.fork(s["src"], s["dst"], s["first"])
        elif kind == "compact":
            s["edit"] = t.compact()
        if kind in ("trim", "sample"):
            s["end"] = t.trim(s["keep"])
        if kind != "trim":
            s["cache"] = KvCache(cfg)
            s["cache"].load(s["codes"], s["exps"])
            del s["codes"], s["exps"]
        if kind in ("diff", "sample"):
            s["max_new"] = max(1, max(s["add"].tolist()))
            s["step"] = t.plan(s["add"], s["limit"], max_new=s["max_new"])
            H, G, D, n = case["heads"], case["group"], case["dim"], s["limit"]
            s["out"] = torch.empty(n, H // 2 * G, 2 * D, dtype=DTYPE[case["dtype"]], device="cuda")
            s["lse"] = torch.empty(n, H * G, device="cuda") if case["lse"] else None
    return s


# ---- one pass -----------------------------------------------------------------------------------------------------

def run(state):
    kind = state["case"]["kind"]
    return (_run_own if own else _run_plain)(state, kind)


def _run_own(s, kind):
    t = s["tables"]
    if kind == "trim":
        return _edit_outputs(t.trim(s["keep"], edit=s["end"]), ring=t.ring)
    cache = s["cache"]
    if kind == "compact":
        t.compact(edit=s["edit"])
        cache.copy(s["edit"])
        return _edit_outputs(s["edit"], moves=s["edit"].moves, kv=cache.export(s["wanted"], DTYPE[s["case"]["dtype"]]))
    if kind in ("fork", "sample"):
        t.fork(s["src"], s["dst"], s["first"], edit=s["edit"])
        cache.copy(s["edit"])
    if kind == "fork":
        return _edit_outputs(s["edit"], moves=s["edit"].moves, granted=s["edit"].granted, table=t.table,
                             kv=cache.export(s["wanted"], DTYPE[s["case"]["dtype"]]))
    if kind == "sample":
        t.commit(s["edit"])
        t.plan(s["add"], s["limit"], max_new=s["max_new"], step=s["step"])
        cache.append(s["step"], s["k"], s["v"])
    cache.attend_diff(t, s["step"], s["q"], s["lam"], weight=s["weight"], gain=GAIN, eps=EPS, out=s["out"],
                      lse=s["lse"], scale=s["scale"])
    if kind == "sample":
        t.commit(s["step"])
        t.commit(t.trim(s["keep"], edit=s["end"]))
    n = s["tokens"]
    return (s["out"][:n], s["lse"][:n]) if s["lse"] is not None else (s["out"][:n],)


def _edit_outputs(edit, **more):
    return dict(lengths=edit.lengths, counters=edit.counters, **more)


def _run_plain(s, kind):
    case = s["case"]
    if kind == "trim":
        return _trim(s, case["page"])
    if kind == "compact":
        e = _compact(s)
        _copy(s, e["moves"])
        return dict(e, kv=_export(s, s["wanted"], case))
    if kind == "diff":
        return _attend(s, s["table"], case)
    e = _fork(s, case["page"])
    _copy(s, e["moves"])
    if kind == "fork":
        return dict(e, kv=_export(s, s["wanted"], case))
    table = _append(s, e, case)
    return _attend(s, table, case)


# ---- the plain forms ----------------------------------------------------------------------------------------------

def _counters(head, free, extra, refused, taken, given, moves, kind):
    return torch.stack([torch.as_tensor(x, device="cuda").long() for x in (head, free, extra, refused, taken, given, moves,
                                                                          kind)]).to(torch.int32)


def _fork(s, page):
    """Lengths, table, moves and counters after the forks."""
    past, src, dst, rows, pool = s["past"].long(), s["src"].long(), s["dst"].long(), s["rows"], s["pool"]
    n_free = s["free"].numel()
    named = torch.bincount(dst, minlength=rows)
    take = torch.minimum(s["first"].long(), past[src])
    ask = torch.where((src != dst) & (past[dst] == 0) & (named[dst] == 1) & (take > 0), take, torch.zeros_like(take))
    full = ask // page
    need = (ask % page > 0).long()
    cum = torch.cumsum(need, 0)
    ok = (ask > 0) & ((need == 0) | (cum <= n_free))
    granted = torch.where(ok, ask, torch.zeros_like(ask))
    fresh = ok & (need > 0)
    ring = torch.cat([s["free"], s["free"].new_zeros(1)])
    new = torch.where(fresh, ring[(cum - 1).clamp(0, n_free)].long(), torch.full_like(cum, -1))
    old = torch.where(fresh, s["table"][src, full.clamp(max=s["width"] - 1)].long(), torch.full_like(cum, -1))
    table = s["table"].clone()
    j, col = ok.nonzero()[:, 0], torch.arange(s["width"], device="cuda")[None, :]
    row = torch.where(col < full[j][:, None], table[src[j]], table[dst[j]])
    row = torch.where((col == full[j][:, None]) & fresh[j][:, None], new[j][:, None].to(torch.int32), row)
    table[dst[j]] = row
    lengths = past.clone()
    lengths[dst[j]] = granted[j]
    taken, zero = fresh.sum(), torch.zeros_like(cum[0])
    return dict(lengths=lengths.to(torch.int32), granted=granted.to(torch.int32), table=table,
                moves=torch.stack([old, new], 1).to(torch.int32),
                counters=_counters(taken % pool, n_free - taken, torch.where(ok, full, zero).sum(),
                                   (~ok).sum(), taken, 0, dst.numel(), 1))


def _trim(s, page):
    """Lengths, ring and counters after requests have let tokens go."""
    past, keep, pool, width = s["past"].long(), s["keep"].long(), s["pool"], s["width"]
    n_free = s["free"].numel()
    col = torch.arange(width, device="cuda")[None, :]
    held = (past + page - 1) // page
    owners = torch.bincount(s["table"][col < held[:, None]].long(), minlength=pool)
    to = torch.where((keep >= 0) & (keep < past), keep, past)
    last = torch.gather(s["table"], 1, (to // page).clamp(max=width - 1)[:, None])[:, 0].long()
    refused = (to < past) & (to % page > 0) & (owners[last] > 1)
    after = torch.where(refused, past, to)
    gone = (col >= ((after + page - 1) // page)[:, None]) & (col < held[:, None])
    ids = s["table"][gone].long()
    count = torch.bincount(ids, minlength=pool)
    at = torch.arange(ids.numel(), device="cuda")
    final = torch.full((pool,), -1, device="cuda").scatter_reduce_(0, ids, at, "amax")
    push = (count[ids] == owners[ids]) & (final[ids] == at)
    given = push.sum()
    ring = torch.zeros(pool, dtype=torch.int32, device="cuda")
    ring[:n_free] = s["free"]
    ring[((n_free - 1 + torch.cumsum(push, 0)) % pool)[push]] = ids[push].to(torch.int32)
    extra = (owners - 1).clamp(min=0).sum() - (ids.numel() - given)
    return dict(lengths=after.to(torch.int32), ring=ring,
                counters=_counters(0, n_free + given, extra, refused.sum(), 0, given, 0, 2))


def _compact(s):
    """Moves and counters of held pages going to the pool's lower end."""
    pool, n_free = s["pool"], s["free"].numel()
    live = torch.ones(pool, dtype=torch.bool, device="cuda")
    live[s["free"].long()] = False
    n = pool - n_free
    src, dst = live[n:].nonzero()[:, 0] + n, (~live[:n]).nonzero()[:, 0]
    moves = torch.full((max(1, pool // 2), 2), -1, dtype=torch.int32, device="cuda")
    moves[:src.numel()] = torch.stack([src, dst], 1).to(torch.int32)
    return dict(lengths=s["past"], moves=moves,
                counters=_counters(n % pool, n_free, 0, 0, 0, 0, src.numel(), 3))


def _copy(s, moves):
    moves = moves.long()
    moves = moves[moves[:, 0] >= 0]
    s["codes"][moves[:, 1]] = s["codes"][moves[:, 0]]
    s["exps"][moves[:, 1]] = s["exps"][moves[:, 0]]


def _export(s, slots, case):
    ids, off = slots // case["page"], slots % case["page"]
    x = _decode(s["codes"][ids, :, :, off], case["form"]) * _pow2(s["exps"][ids])[..., None]
    x = x.to(DTYPE[case["dtype"]])
    return x[:, :, 0].contiguous(), x[:, :, 1].contiguous()


def _append(s, e, case):
    """One new token for each fork: its slot, and its keys and values in the cache.  Returns the table."""
    form, page, H, codes, exps = case["form"], case["page"], case["heads"], s["codes"], s["exps"]
    table, R = e["table"], case["R"]
    past = e["lengths"].long()[R:]
    off, n = past % page, past // page
    fresh = off == 0
    at = e["counters"][4] + torch.cumsum(fresh.long(), 0) - 1
    row = torch.arange(R, s["rows"], device="cuda")
    ids = torch.where(fresh, s["free"][at.clamp(min=0)], table[row, n]).long()
    table[row, n] = ids.to(torch.int32)
    x = torch.stack([s["k"][:s["tokens"]].float(), s["v"][:s["tokens"]].float()], 2)           # [n][H][2][D]
    need, before = _need(x.abs().amax(-1), form), exps[ids]
    after = torch.where(fresh[:, None, None], need, torch.maximum(before, need))
    codes[ids] = _encode(_decode(codes[ids], form) * _pow2(torch.clamp(before - after, max=0))[..., None, None], form)
    exps[ids] = after
    codes[ids, :, :, off] = _encode(x * _pow2(-after)[..., None], form)
    return table


def _attend(s, table, case):
    H, G, D, page, form = case["heads"], case["group"], case["dim"], case["page"], case["form"]
    P, n_all = H // 2, s["tokens"]
    out = torch.zeros(n_all, P * G, 2 * D, device="cuda")
    lse = torch.full((n_all, H * G), float("-inf"), device="cuda")
    lam = s["lam"].expand(s["limit"], P * G)
    first = 0
    for i, past, n in _window(case):
        L = past + n
        ids = table[i, :_pages(L, page)].long()
        kv = _decode(s["codes"][ids], form) * _pow2(s["exps"][ids])[..., None, None]   # [pages][H][2][page][D]
        kt = kv[:, :, 0].permute(1, 3, 0, 2).reshape(H, D, -1)[:, :, :L].contiguous()
        v = kv[:, :, 1].unflatten(1, (P, 2)).permute(1, 0, 3, 2, 4).reshape(P, -1, 2 * D)[:, :L].contiguous()
        rows = max(1, min(n, (1 << 28) // (H * G * L)))
        for a in range(first, first + n, rows):
            b = min(first + n, a + rows)
            q = s["q"][a:b].float().unflatten(1, (H, G)).permute(1, 0, 2, 3).reshape(H, -1, D)
            sc = torch.bmm(q, kt) * s["scale"]                                        # [H][rows * G][L]
            if n > 1:
                last = past + torch.arange(a - first, b - first, device="cuda").repeat_interleave(G)
                sc = sc.masked_fill(torch.arange(L, device="cuda")[None, :] > last[:, None], float("-inf"))
            m = sc.amax(-1, keepdim=True)
            p = torch.exp(sc - m)
            l = p.sum(-1, keepdim=True)
            p = p / l
            la = lam[a:b].unflatten(1, (P, G)).permute(1, 0, 2).reshape(P, -1, 1)
            o = torch.bmm(p[0::2] - la * p[1::2], v)
            out[a:b] = o.unflatten(1, (b - a, G)).permute(1, 0, 2, 3).reshape(b - a, P * G, 2 * D)
            lse[a:b] = (m + torch.log(l))[..., 0].unflatten(1, (b - a, G)).permute(1, 0, 2).reshape(b - a, H * G)
        first += n
    if case["norm"]:
        out = out * torch.rsqrt((out * out).mean(-1, keepdim=True) + EPS) * s["weight"]
    out = (out * GAIN).to(DTYPE[case["dtype"]])
    return (out, lse) if case["lse"] else (out,)


def _window(case):
    """(row, tokens before, new tokens) of the requests with new tokens, as the program knows them on the host."""
    o = _plan_of(case)
    for i, a in enumerate(o["add"]):
        if a > 0:
            yield i, o["past"][i if case["kind"] == "diff" else o["parent"][i]], a


# ---- what a pass cannot do without --------------------------------------------------------------------------------

def work(case):
    o, width, held, pool, tokens = _sizes(case)
    H, G, D, page, kind = case["heads"], case["group"], case["dim"], case["page"], case["kind"]
    rows, wide = len(o["past"]), H * D
    page_bytes = 2 * page * wide + 8 * H
    if kind == "trim":
        keep = [k if 0 <= k < p else p for k, p in zip(o["keep"], o["past"])]
        gone = sum(_pages(p, page) - _pages(k, page) for k, p in zip(keep, o["past"]))
        return {"bytes": 12 * rows + 12 * gone, "flops": 4 * rows + 4 * gone}
    if kind == "compact":
        moves = _moves(held, pool)
        return {"bytes": 8 * (pool - held) + 8 * moves + moves * (2 * page_bytes + page * wide * 2 * (1 + 2)),
                "flops": pool + 2 * moves * page * wide}
    fork_bytes = copies = 0
    if kind in ("fork", "sample"):
        copies = sum(t % page > 0 for t in o["tokens"])
        fork_bytes = 12 * rows + 20 * len(o["dst"]) + 8 * sum(t // page for t in o["tokens"]) + 2 * copies * page_bytes
    if kind == "fork":
        return {"bytes": fork_bytes + copies * page * wide * 2 * (1 + 2), "flops": 10 * len(o["dst"]) + 2 * copies * page * wide}
    lengths = [p for _, p, _ in _window(case)], [a for _, _, a in _window(case)]
    keys = sum(a * p + a * (a + 1) // 2 for p, a in zip(*lengths))
    if kind == "sample":
        # a family's shared pages are read once; the new tokens' own page, for each
        tokens_read = sum(o["past"][:case["R"]]) + tokens * page
    else:
        tokens_read = sum(p + a for p, a in zip(*lengths))
    attend = tokens_read * wide * 2 + _pages(tokens_read, page) * H * 8 + tokens * wide * G * 2 * 2
    if kind == "sample":
        attend += tokens * wide * 2 * 3 + 12 * rows
    # a key of a row: two maps' scores, 2 dim each, and their sums over 2 dim numbers, 4 dim each
    return {"bytes": fork_bytes + attend, "flops": 12 * D * H // 2 * G * keys}


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


def _exact_fork(case, s):
    o, width, held, pool, _ = _sizes(case)
    page, free, table, lengths = case["page"], s["free"].tolist(), s["table"].tolist(), list(o["past"])
    granted, moves, asked, shared, refused = [], [], 0, 0, 0
    for j, (a, b, t) in enumerate(zip(o["src"], o["dst"], o["tokens"])):
        t = min(t, o["past"][a])
        if a == b or o["past"][b] or o["dst"].count(b) > 1 or t <= 0:
            t = 0
        asked += t % page > 0
        ok = t > 0 and (t % page == 0 or asked <= len(free))
        granted.append(t if ok else 0)
        moves.append((-1, -1))
        refused += not ok
        if ok:
            shared += t // page
            table[b][:t // page] = s_row = table[a][:t // page]
            lengths[b] = t
            if t % page:
                moves[-1] = table[a][len(s_row)], free[asked - 1]
                table[b][len(s_row)] = free[asked - 1]
    taken = sum(m[0] >= 0 for m in moves)
    return dict(lengths=_i32(lengths), granted=_i32(granted), table=_i32(table), moves=_i32(moves),
                counters=_i32([taken % pool, len(free) - taken, shared, refused, taken, 0, len(moves), 1]))


def _exact_trim(case, s):
    o, width, held, pool, _ = _sizes(case)
    page, free, table = case["page"], s["free"].tolist(), s["table"].tolist()
    owners, goes, lengths, refused = [0] * pool, [0] * pool, [], 0
    for i, p in enumerate(o["past"]):
        for n in range(_pages(p, page)):
            owners[table[i][n]] += 1
    for i, (p, k) in enumerate(zip(o["past"], o["keep"])):
        k = k if 0 <= k < p else p
        if k < p and k % page and owners[table[i][k // page]] > 1:
            k, refused = p, refused + 1
        lengths.append(k)
        for n in range(_pages(k, page), _pages(p, page)):
            goes[table[i][n]] += 1
    left, back = list(goes), []
    for i, (p, k) in enumerate(zip(o["past"], lengths)):
        for n in range(_pages(k, page), _pages(p, page)):
            g = table[i][n]
            left[g] -= 1
            if left[g] == 0 and goes[g] == owners[g]:
                back.append(g)
    ring = (free + back + [0] * pool)[:pool]
    extra = sum(max(0, a - b - 1) for a, b in zip(owners, goes))
    return dict(lengths=_i32(lengths), ring=_i32(ring),
                counters=_i32([0, len(free) + len(back), extra, refused, 0, len(back), 0, 2]))


def _exact_compact(case, s):
    pool, free = s["pool"], set(s["free"].tolist())
    n = pool - len(free)
    moves = list(zip((p for p in range(n, pool) if p not in free), (p for p in range(n) if p in free)))
    rest = [(-1, -1)] * (max(1, pool // 2) - len(moves))
    return dict(lengths=s["past"], moves=_i32(moves + rest), counters=_i32([n % pool, len(free), 0, 0, 0, 0, len(moves), 3]))


def exact(case, seed):
    s = _inputs(case, seed)
    kind, page, form = case["kind"], case["page"], case["form"]
    if kind == "trim":
        return _exact_trim(case, s)
    if kind in ("fork", "compact"):
        e = _exact_fork(case, s) if kind == "fork" else _exact_compact(case, s)
        ids = torch.tensor([a for a, _ in e["moves"].tolist() if a >= 0], dtype=torch.long, device="cuda")
        if ids.numel() * page * case["heads"] * case["dim"] > 1 << 29:
            return dict(e, kv=(None, None))     # (64 bits of that many numbers are beyond a few seconds)
        x = _values64(s["codes"][ids], form) * torch.exp2(s["exps"][ids].double())[..., None, None]
        x = x.permute(0, 3, 1, 2, 4).flatten(0, 1)
        return dict(e, kv=(x[:, :, 0].contiguous(), x[:, :, 1].contiguous()))
    H, G, D = case["heads"], case["group"], case["dim"]
    P, tokens = H // 2, s["tokens"]
    table = s["table"].tolist()
    out = torch.zeros(tokens, P * G, 2 * D, dtype=torch.float64, device="cuda")
    lse = torch.full((tokens, H * G), float("-inf"), dtype=torch.float64, device="cuda")
    first = 0
    for i, past, n in _window(case):
        L = past + n
        ids = torch.tensor((table[i] if kind == "diff" else table[i % case["R"]])[:_pages(past + (n if kind == "diff" else 0), page)],
                           dtype=torch.long, device="cuda")
        for p in range(P):
            kv = _values64(s["codes"][ids, 2 * p:2 * p + 2], form) * torch.exp2(s["exps"][ids, 2 * p:2 * p + 2].double())[..., None, None]
            kv = kv.permute(1, 2, 0, 3, 4).flatten(2, 3)                               # [2][2][tokens][D]
            if kind == "sample":
                kv = _with_token(case, s, kv[:, :, :past], first, 2 * p, ids)
            kv = kv[:, :, :L]
            v = torch.cat([kv[0, 1], kv[1, 1]], 1).contiguous()
            for a in range(0, n, 1024):
                b = min(n, a + 1024)
                later = torch.arange(L, device="cuda")[None, :] > torch.arange(past + a, past + b, device="cuda")[:, None]
                for g in range(G):
                    maps = []
                    for z in range(2):
                        hq = (2 * p + z) * G + g
                        sc = s["q"][first + a:first + b, hq].double().contiguous() @ kv[z, 0].t().contiguous() * s["scale"]
                        sc[later] = float("-inf")
                        both = torch.logsumexp(sc, -1)
                        lse[first + a:first + b, hq] = both
                        maps.append(torch.exp(sc - both[:, None]) @ v)
                    la = s["lam"].double().expand(s["limit"], P * G)[first + a:first + b, p * G + g]
                    out[first + a:first + b, p * G + g] = maps[0] - la[:, None] * maps[1]
        first += n
    if case["norm"]:
        out = out / torch.sqrt(out.square().mean(-1, keepdim=True) + EPS) * s["weight"].double()
    out = out * GAIN
    return (out, lse) if case["lse"] else (out,)


def _with_token(case, s, kv, t, h, ids):
    """A fork's keys and values [2][2][tokens][D] of heads h, h + 1 with row t's behind them, as its last page holds
    them: all on the page's scale."""
    page, form, past = case["page"], case["form"], kv.shape[2]
    from_ = past // page * page
    new = torch.stack([s["k"][t, h:h + 2].double(), s["v"][t, h:h + 2].double()], 1)[:, :, None]
    kv = torch.cat([kv, new], 2)
    for z in range(2):
        for side in range(2):
            e = _exponent64(float(new[z, side].abs().max()), form)
            if past % page:
                e = max(e, int(s["exps"][ids[past // page], h + z, side]))
            kv[z, side, from_:] = _round64(kv[z, side, from_:] / 2.0 ** e, form) * 2.0 ** e
    return kv
