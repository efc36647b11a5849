"""The paged cache on the GPU against its 64-bit reference (kv_reference.py).

Tables, slots and stored values are compared exactly: all of them are whole
numbers or numbers with at most eight significant bits.

Attention.  With u the half unit of q's type (2^-9 bf16, 2^-12 fp16) an output
is off by at most u (its own rounding) plus u (each probability's rounding)
times the largest |v| its keys have; a probability in fp16 that is small beside
the largest loses up to 2^-25 of it, per key; a score's products and sums in
fp32 are off by at most (dim + 4) 2^-24 times sum |q k|, which moves every
probability by that share, twice (over the quotient); N keys' sums by
2 N 2^-24.  The logarithm of the sum: the score's part, the sum's part, and
2^-22 of its own size for the exponential and logarithm.
"""
import numpy as np
import pytest
import torch

from gpu_helpers import say
from kv_reference import Node
from paper_2508_01744_amd import AgftError, KvCache, KvStep, KvTables, kv_config

pytestmark = pytest.mark.gpu
T = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def make(requests, row_pages, pages, page=16, heads=2, group=2, dim=64, form="e4m3"):
    cfg = kv_config(requests, row_pages * page, pages, page=page, heads=heads, group=group, dim=dim, form=form)
    return (cfg, KvTables(cfg), KvCache(cfg),
            Node(requests, row_pages, pages, page, heads, group, dim, form))


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def same_plan(tables, step, node, want, max_tokens):
    assert step.starts.tolist() == want["starts"]
    assert step.granted.tolist() == want["granted"]
    assert step.lengths.tolist() == want["lengths"]
    assert step.counters.tolist() == want["counters"]
    assert step.slots.tolist() == want["slots"]
    got = tables.table.cpu().numpy()
    for i, n in enumerate(want["lengths"]):
        used = -(-n // node.page)
        assert (got[i, :used] == node.table[i, :used]).all(), i
    ring = tables.ring.tolist()
    for n in range(want["counters"][1]):
        at = (want["counters"][0] + n) % node.P
        assert ring[at] == node.ring[at]


@pytest.mark.parametrize("requests,row_pages,pages,page,seed", [
    (1, 4, 4, 16, 0), (1, 1, 1, 128, 1), (5, 7, 20, 16, 2), (64, 9, 300, 32, 3), (65, 9, 100, 16, 4),
    (1023, 6, 3000, 16, 5), (1025, 5, 2000, 64, 6), (3000, 4, 5000, 16, 7)])
def test_plan_over_windows(requests, row_pages, pages, page, seed):
    """Many windows of joins, tokens, chunks, ends and refusals."""
    say("plan", requests, row_pages, pages, page, seed)
    rng = np.random.default_rng(seed)
    _, tables, _, node = make(requests, row_pages, pages, page)
    for window in range(12):
        kind = rng.integers(0, 6, requests)
        add = np.select([kind == 0, kind == 1, kind == 2], [0, rng.integers(1, 3 * page, requests),
                                                             rng.integers(-2, 0, requests)], 1)
        if window % 5 == 4:
            add[rng.integers(0, requests)] = row_pages * page + 1      # longer than a row
        asked = int(np.maximum(add, 0).sum())
        max_tokens = max(1, asked + int(rng.integers(-3, 40)))
        step = tables.plan(ints(add.tolist()), max_tokens)
        again = tables.plan(ints(add.tolist()), max_tokens, step=step)   # planning changes no state
        want = node.plan(add.tolist(), max_tokens)
        same_plan(tables, again, node, want, max_tokens)
        tables.commit(step)
        node.commit(want)
        live = [int(p) for i in range(requests) for p in node.table[i, :-(-node.lengths[i] // page)]]
        assert len(live) == len(set(live)) and len(live) + node.free == pages


def test_plan_refuses_what_does_not_fit():
    """A full pool still serves requests that have room in their last page."""
    _, tables, _, node = make(4, 4, 5, 16)
    for add in ([17, 17, 16, 0], [1, 1, 1, 1], [15, 14, 1, 5], [0, -1, 0, 0], [1, 30, 1, 33], [-1, 1, -7, 2]):
        step = tables.plan(ints(add), 64)
        want = node.plan(add, 64)
        same_plan(tables, step, node, want, 64)
        tables.commit(step)
        node.commit(want)


def test_plan_at_the_largest_lengths():
    """Sums of what is asked that pass 32 bits, and a limit that cuts them."""
    rows = (1 << 30) // 128 - 1
    cfg = kv_config(3, rows * 128, 64, page=128, heads=1, group=1, dim=64)
    tables = KvTables(cfg)
    top = rows * 128
    step = tables.plan(ints([top, top, 130]), 200)
    assert step.granted.tolist() == [0, 0, 0] and step.starts.tolist() == [0, 200, 200, 200]
    assert step.counters.tolist()[2:6] == [200, 3, 0, 0] and set(step.slots.tolist()) == {-1}
    step = tables.plan(ints([0, -1, 130]), 200)
    assert step.granted.tolist() == [0, 0, 130] and step.slots.tolist()[:130] == list(range(130))


def window_tensors(rng, n, heads, dim, dtype, wide=True):
    """A [n][heads][dim] view into a wider tensor, near normal with rows of very
    different size, and the same numbers in 64 bits."""
    pad = 16 if wide else 0
    x = rng.standard_normal((n, heads * dim + pad)) * np.exp2(rng.integers(-6, 7, (n, 1)))
    t = torch.tensor(x, device="cuda").to(dtype)
    view = t[:, pad:].unflatten(1, (heads, dim))
    return view, view.double().cpu().numpy()


APPENDS = [(page, dim, form, dtype) for page, dim in ((16, 64), (32, 128), (64, 256), (128, 64), (128, 128))
           for form, dtype in (("e4m3", "bf16"), ("int8", "fp16"), ("int8", "fp32"), ("e4m3", "fp32"))]


@pytest.mark.parametrize("page,dim,form,dtype", APPENDS)
def test_append_and_export(page, dim, form, dtype):
    """Windows of single tokens and chunks, pages that fill over several of them
    with exponents that rise, odd starts."""
    say("append", page, dim, form, dtype)
    rng = np.random.default_rng(page + dim)
    _, tables, cache, node = make(5, 4, 18, page, heads=3, dim=dim, form=form)
    for add in ([1, page, page + 1, 5, 0], [1, 1, 2, page - 5, 3], [3, 0, page - 3, 1, 1], [1, 1, -1, 1, 2 * page]):
        n = max(1, sum(max(a, 0) for a in add)) + 2
        step = tables.plan(ints(add), n)
        want = node.plan(add, n)
        k, k64 = window_tensors(rng, n, 3, dim, T[dtype])
        v, v64 = window_tensors(rng, n, 3, dim, T[dtype])
        cache.append(step, k, v)
        node.append(want, k64, v64)
        tables.commit(step)
        node.commit(want)
        slots = [int(node.table[i, t // page]) * page + t % page for i in range(5) for t in range(node.lengths[i])]
        slots += [-1, node.P * page, slots[0]]          # nothing there, past the pool, a slot twice
        ref = node.export([s if s < node.P * page else -1 for s in slots])
        for out in (torch.float32, T[dtype]):
            gk, gv = cache.export(torch.tensor(slots, device="cuda"), out)
            assert gk.shape == gv.shape == (len(slots), 3, dim) and gk.dtype == out
            assert (gk.double().cpu().numpy() == ref[:, :, 0]).all()
            assert (gv.double().cpu().numpy() == ref[:, :, 1]).all()
    assert cache.export(torch.empty(0, dtype=torch.int64, device="cuda"))[0].shape == (0, 3, dim)


@pytest.mark.parametrize("form", ["e4m3", "int8"])
def test_append_of_unusual_numbers(form):
    """Zeros, the smallest and largest numbers, infinities, NaN, exact ends of a
    code's range, and a page whose exponent rises all the way."""
    _, tables, cache, node = make(1, 2, 2, 16, heads=1, dim=64, form=form)
    top = 3e38      # (what rounds past fp32's largest number has no fp32 value to come back as)
    rows = [np.zeros(64), np.full(64, 2.0 ** -149), np.full(64, 1e-30), np.linspace(-1, 1, 64),
            np.full(64, 448.0), np.full(64, 127.0), np.array([np.inf, -np.inf, np.nan, 3.0] * 16),
            np.full(64, np.nan), np.full(64, -top), np.linspace(-2.0, 1.5, 64), np.full(64, np.inf)]
    rng = np.random.default_rng(5)
    for x in rows + [rng.standard_normal((7, 64)), np.full((3, 64), 7.0)]:
        x = np.atleast_2d(np.asarray(x, dtype=np.float32))
        n = x.shape[0]
        step, want = tables.plan(ints([n]), n), node.plan([n], n)
        t = torch.tensor(x[:, None, :], device="cuda")
        cache.append(step, t, torch.flip(t, [2]).contiguous())
        x64 = x[:, None, :].astype(np.float64)
        node.append(want, x64, x64[:, :, ::-1])
        tables.commit(step)
        node.commit(want)
        slots = [int(node.table[0, j // 16]) * 16 + j % 16 for j in range(node.lengths[0])]
        # an infinity beside 3e38 is held as 448 (or 127) 2^120 and more, which fp32 gives back as infinity
        with np.errstate(over="ignore"):
            ref = node.export(slots).astype(np.float32)
        gk, gv = cache.export(torch.tensor(slots, device="cuda"), torch.float32)
        assert (gk.double().cpu().numpy() == ref[:, :, 0]).all()
        assert (gv.double().cpu().numpy() == ref[:, :, 1]).all()


def attend_and_compare(tables, cache, node, step, want, rng, dtype, scale=None, lse=True, tell=""):
    n = step.max_tokens
    hq = node.H * node.G
    q, q64 = window_tensors(rng, n, hq, node.D, T[dtype])
    q = q / q.float().abs().amax(-1, keepdim=True).clamp(min=1.0).to(q.dtype) * 2      # scores of a few units
    q64 = q.double().cpu().numpy()
    out = torch.full((n, hq, node.D), 7.0, dtype=T[dtype], device="cuda")
    sums = torch.full((n, hq), 7.0, device="cuda") if lse else None
    cache.attend(tables, step, q, out=out, lse=sums, scale=scale)
    s = node.D ** -0.5 if scale is None else scale
    ref, ref_lse, vmax, smax, keys = node.attend(want, q64[:want["starts"][-1]], s)
    rows = want["starts"][-1]
    got = out[:rows].double().cpu().numpy()
    u = 2.0 ** -9 if dtype == "bf16" else 2.0 ** -12
    small = keys * 2.0 ** -25 if dtype == "fp16" else 0.0
    score = (node.D + 4) * 2.0 ** -24 * smax
    tol = (2 * u + small + 2 * score + 4 * keys * 2.0 ** -24) * vmax + 1e-30
    err = np.abs(got - ref).max(-1, initial=0.0)
    worst = float((err / tol).max(initial=0.0))
    assert (err <= tol).all(), (tell, worst, np.argwhere(err > tol)[:4].tolist())
    if lse:
        g = sums[:rows].double().cpu().numpy()
        empty = np.isinf(ref_lse)
        assert (np.isneginf(g) == empty).all()
        off = np.abs(g - ref_lse)[~empty]
        assert (off <= (score + 2 * keys * 2.0 ** -24 + 2.0 ** -22 * (1 + np.abs(ref_lse)))[~empty]).all(), off.max()
        assert (sums[rows:] == 7.0).all()
    assert (out[rows:] == 7.0).all()          # rows past the window's tokens are left alone
    return worst


def fill(tables, cache, node, rng, add, dtype):
    n = max(1, sum(max(a, 0) for a in add)) + 3
    step, want = tables.plan(ints(add), n, max_new=max(1, max(add))), node.plan(add, n)
    k, k64 = window_tensors(rng, n, node.H, node.D, T[dtype])
    v, v64 = window_tensors(rng, n, node.H, node.D, T[dtype])
    cache.append(step, k, v)
    node.append(want, k64, v64)
    return step, want


HEADS = [  # heads, group, dim, page, form, dtype
    (2, 4, 64, 16, "e4m3", "bf16"), (1, 1, 128, 16, "int8", "fp16"), (3, 5, 128, 32, "e4m3", "fp16"),
    (1, 16, 64, 64, "int8", "bf16"), (2, 3, 256, 16, "e4m3", "bf16"), (1, 8, 256, 128, "int8", "fp16"),
    (1, 40, 64, 16, "e4m3", "bf16"), (4, 1, 64, 128, "int8", "fp16"), (1, 128, 128, 32, "int8", "bf16")]


@pytest.mark.parametrize("heads,group,dim,page,form,dtype", HEADS)
def test_attend_single_tokens(heads, group, dim, page, form, dtype):
    """One token per request over caches of 1 to some hundred tokens, ends of
    blocks, pages and units of work among them; idle and ended requests beside."""
    say("attend single", heads, group, dim, page, form, dtype)
    rng = np.random.default_rng(dim + page + group)
    lengths = [0, 1, 14, 15, 16, 17, 31, 62, 63, 64, 65, 127, 128, 300, 511]
    _, tables, cache, node = make(len(lengths) + 2, 1024 // page, (4096 + 64 * page) // page, page, heads, group, dim, form)
    step, want = fill(tables, cache, node, rng, lengths + [9, 9], dtype)
    tables.commit(step)
    node.commit(want)
    step, want = fill(tables, cache, node, rng, [1] * len(lengths) + [0, -1], dtype)
    worst = attend_and_compare(tables, cache, node, step, want, rng, dtype)
    say("  worst share of the bound", worst)


@pytest.mark.parametrize("heads,group,dim,page,form,dtype", HEADS)
def test_attend_chunks(heads, group, dim, page, form, dtype):
    """Prompts and chunks of many lengths beside single tokens, with and without
    tokens held before."""
    say("attend chunks", heads, group, dim, page, form, dtype)
    rng = np.random.default_rng(dim + 3 * page + group)
    scale = 4 if group > 30 else 1
    adds = [[1, 2, 3, 40 // scale, 0, 16, 5], [1, 70 // scale, 2, 130 // scale, 33 // scale, 1, 0], [1, 1, 4, 17, 64 // scale, -1, 3]]
    _, tables, cache, node = make(7, 512 // page, 3584 // page, page, heads, group, dim, form)
    for add in adds:
        step, want = fill(tables, cache, node, rng, add, dtype)
        worst = attend_and_compare(tables, cache, node, step, want, rng, dtype)
        say("  worst share of the bound", worst)
        tables.commit(step)
        node.commit(want)


@pytest.mark.parametrize("dim,dtype,form", [(128, "bf16", "e4m3"), (64, "fp16", "int8")])
def test_attend_long_and_split(dim, dtype, form):
    """Few rows over a long cache, which is shared out and joined, beside short
    ones; a chunk at its end."""
    rng = np.random.default_rng(dim)
    _, tables, cache, node = make(4, 640, 900, 16, 1, 4, dim, form)
    step, want = fill(tables, cache, node, rng, [9000, 3, 1500, 0], dtype)
    tables.commit(step)
    node.commit(want)
    for add in ([1, 1, 1, 1], [2, 1, 30, 5]):
        step, want = fill(tables, cache, node, rng, add, dtype)
        say("  worst share of the bound", attend_and_compare(tables, cache, node, step, want, rng, dtype))
        tables.commit(step)
        node.commit(want)


def test_attend_of_refused_tokens():
    """Tokens without slots: rows of zeros and logarithms of nothing, for single
    tokens and for chunks, and the others as ever."""
    rng = np.random.default_rng(9)
    _, tables, cache, node = make(5, 8, 6, 16, 2, 4, 64, "e4m3")
    step, want = fill(tables, cache, node, rng, [16, 16, 20, 0, 3], "bf16")
    assert want["granted"] == [16, 16, 20, 0, 3]
    tables.commit(step)
    node.commit(want)
    for add in ([1, 1, 1, 1, 1], [40, 1, 3, 20, 4]):
        step, want = fill(tables, cache, node, rng, add, "bf16")
        assert 0 in [g for g, a in zip(want["granted"], add) if a]
        attend_and_compare(tables, cache, node, step, want, rng, "bf16")


def test_attend_ignores_what_lies_beyond_the_lengths():
    """Codes of NaN in unused tokens, in pages of nobody, and wild table entries
    behind a row's pages change no bit."""
    rng = np.random.default_rng(11)
    outs = []
    for poison in (0, 0x7F):
        r = np.random.default_rng(3)
        _, tables, cache, node = make(3, 16, 40, 32, 1, 4, 128, "e4m3")
        cache.codes.fill_(poison)
        tables.table.fill_(0 if poison == 0 else 2 ** 31 - 1)
        for add in ([70, 5, 33], [1, 1, 1], [20, 1, 3]):
            step, want = fill(tables, cache, node, r, add, "bf16")
            q, _ = window_tensors(np.random.default_rng(8), step.max_tokens, 4, 128, torch.bfloat16)
            o = cache.attend(tables, step, q)[:want["starts"][-1]]
            assert torch.isfinite(o).all()
            outs.append(o.clone())
            tables.commit(step)
            node.commit(want)
    for a, b in zip(outs[:3], outs[3:]):
        assert torch.equal(a, b)


def test_scale_of_pages_far_apart():
    """Pages whose exponents lie far apart: the small ones' part is not lost, the
    large ones' does not overflow fp16's probabilities."""
    rng = np.random.default_rng(2)
    for dtype, step_size in (("fp16", 2.0 ** -4), ("bf16", 2.0 ** -12)):
        _, tables, cache, node = make(2, 16, 32, 16, 1, 2, 64, "e4m3")
        for w in range(6):
            n = 34
            add = [16, 16]
            step, want = tables.plan(ints(add), n), node.plan(add, n)
            x = rng.standard_normal((2, n, 1, 64))
            k, v = (torch.tensor(z * f, device="cuda").to(T[dtype]) for z, f in
                    zip(x, (1.0, (step_size ** (w if w < 3 else 5 - w)) * 8)))
            cache.append(step, k, v)
            node.append(want, k.double().cpu().numpy(), v.double().cpu().numpy())
            attend_and_compare(tables, cache, node, step, want, rng, dtype)
            tables.commit(step)
            node.commit(want)


def test_nan_in_one_query_stays_in_its_row():
    rng = np.random.default_rng(4)
    _, tables, cache, node = make(2, 16, 32, 16, 1, 4, 64, "int8")
    step, want = fill(tables, cache, node, rng, [50, 1], "bf16")
    q, _ = window_tensors(rng, step.max_tokens, 4, 64, torch.bfloat16)
    q = q.contiguous()
    clean = cache.attend(tables, step, q).clone()
    q[7, 2, 5] = float("nan")
    q[50, 1, 0] = float("nan")
    out = cache.attend(tables, step, q)
    bad = torch.isnan(out).any(-1)[:51]
    assert bad.sum() == 2 and bad[7, 2] and bad[50, 1]
    assert torch.equal(out[:51][~bad], clean[:51][~bad])


def test_offsets_past_32_bits():
    """A cache of more than 4 GiB: the last pages hold and give what they should."""
    pages = (9 << 29) // (2 * 128 * 8 * 256)      # 4.5 GiB
    cfg = kv_config(2, 512, pages, page=128, heads=8, group=1, dim=256)
    tables, cache = KvTables(cfg), KvCache(cfg)
    table = torch.zeros(2, 4, dtype=torch.int32, device="cuda")
    free = torch.tensor([pages - 1, pages - 2, 0, 1], dtype=torch.int32, device="cuda")
    tables.load(torch.zeros(2, dtype=torch.int32, device="cuda"), table, free)
    node = Node(2, 4, 4, 128, 8, 1, 256, "e4m3")
    order = {0: pages - 1, 1: pages - 2, 2: 0, 3: 1}
    rng = np.random.default_rng(1)
    step, want = fill(tables, cache, node, rng, [130, 20], "bf16")
    assert step.slots.tolist()[:150] == [order[s // 128] * 128 + s % 128 for s in want["slots"][:150]]
    attend_and_compare(tables, cache, node, step, want, rng, "bf16")
    gk, _ = cache.export(step.slots[:150].contiguous(), torch.float32)
    assert (gk.double().cpu().numpy() == node.export(want["slots"][:150])[:, :, 0]).all()


def test_streams_and_graphs():
    """On a stream of its own, and recorded into a graph of several windows that
    is replayed, with eager work between, against eager calls."""
    rng = np.random.default_rng(6)
    cfg, tables, cache, node = make(4, 16, 64, 16, 2, 4, 64, "e4m3")
    step, want = fill(tables, cache, node, rng, [40, 3, 17, 1], "bf16")
    tables.commit(step)
    node.commit(want)
    ones = ints([1, 1, 1, 1])
    k, k64 = window_tensors(rng, 4, 2, 64, torch.bfloat16)
    q, _ = window_tensors(rng, 4, 8, 64, torch.bfloat16)
    step = KvStep(cfg, 4, 1)
    out = torch.empty(4, 8, 64, dtype=torch.bfloat16, device="cuda")

    def window(tb, ch):
        tb.plan(ones, 4, max_new=1, step=step)
        ch.append(step, k, k)
        ch.attend(tb, step, q, out=out)
        tb.commit(step)

    twin_t, twin_c = KvTables(cfg), KvCache(cfg)
    twin_t.buffer.copy_(tables.buffer)
    twin_c.buffer.copy_(cache.buffer)
    step.work()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        window(tables, cache)
    for _ in range(20):
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        window(twin_t, twin_c)
        torch.cuda.synchronize()
        assert torch.equal(out, got)
        assert torch.equal(twin_t.lengths, tables.lengths) and torch.equal(twin_t.counters[:2], tables.counters[:2])
    # an explicit stream
    twin_t.set_stream(side)
    twin_c.set_stream(side)
    window(twin_t, twin_c)
    side.synchronize()
    got = out.clone()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, got)


def test_equal_calls_give_equal_bits():
    rng = np.random.default_rng(12)
    _, tables, cache, node = make(6, 400, 900, 16, 2, 4, 128, "e4m3")
    step, want = fill(tables, cache, node, rng, [5000, 700, 3, 1, 90, 16], "bf16")
    q, _ = window_tensors(rng, step.max_tokens, 8, 128, torch.bfloat16)
    first = cache.attend(tables, step, q).clone()
    for _ in range(3):
        assert torch.equal(cache.attend(tables, step, q)[:want["starts"][-1]], first[:want["starts"][-1]])


def test_front_end_refuses():
    cfg, tables, cache, _ = make(2, 4, 8, 16, 2, 4, 64)
    dev = "cuda"
    add = ints([3, 1])
    with pytest.raises(ValueError):
        kv_config(2, 64, 8, form="e5m2")
    for bad in (add.long(), add[:1], add.cpu(), ints([1, 2, 3, 4])[::2]):
        with pytest.raises(ValueError):
            tables.plan(bad, 8)
    for n in (0, -1, (1 << 30) + 1):
        with pytest.raises(ValueError):
            tables.plan(add, n)
    with pytest.raises(ValueError):
        tables.plan(add, 8, max_new=9)
    step = tables.plan(add, 8)
    with pytest.raises(ValueError):
        tables.plan(add, 9, step=step)
    k = torch.zeros(8, 2, 64, dtype=torch.bfloat16, device=dev)
    for bad in (k[:7], k.cpu(), k.double(), k[:, :1], torch.zeros(8, 2, 128, dtype=torch.bfloat16, device=dev),
                torch.zeros(8, 2, 65, dtype=torch.bfloat16, device=dev)[:, :, 1:],
                torch.zeros(8, 2, 128, dtype=torch.bfloat16, device=dev)[:, :, ::2]):
        with pytest.raises(ValueError):
            cache.append(step, bad, bad)
    with pytest.raises(ValueError):
        cache.append(step, k, k.half())
    q = torch.zeros(8, 8, 64, dtype=torch.bfloat16, device=dev)
    with pytest.raises(ValueError):
        cache.attend(tables, step, q.float())
    with pytest.raises(ValueError):
        cache.attend(tables, step, q[:, :6])
    with pytest.raises(ValueError):
        cache.attend(tables, step, q, out=q.half())
    with pytest.raises(ValueError):
        cache.attend(tables, step, q, lse=torch.zeros(8, 7, device=dev))
    with pytest.raises(AgftError):
        cache.attend(tables, step, q, scale=float("nan"))
    for bad in (add, torch.zeros(2, 2, dtype=torch.int64, device=dev), torch.zeros(4, dtype=torch.int64)):
        with pytest.raises(ValueError):
            cache.export(bad)
    with pytest.raises(ValueError):
        cache.export(torch.zeros(1, dtype=torch.int64, device=dev), torch.float64)
    with pytest.raises(ValueError):
        tables.load(add, tables.table.clone(), ints([8]))
    with pytest.raises(ValueError):
        tables.load(ints([0, 65]), tables.table.clone(), ints([0]))
    for kw in (dict(dim=96), dict(page=24), dict(heads=0), dict(group=129), dict(pages=0)):
        args = dict(requests=2, row_tokens=64, pages=8)
        args.update(kw)
        with pytest.raises(ValueError):
            KvTables(kv_config(**args))
    torch.cuda.synchronize()
