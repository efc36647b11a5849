"""Differential attention on the GPU against diff_reference.py, at sizes, masks and
layouts where it can go wrong; the bound is derived there."""
import pytest
import torch

from diff_reference import compare, lambdas, reference, weights
from gpu_helpers import say
from kv_flat import Window
from paper_2508_01744_amd import KvCache, KvTables, kv_config

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("form", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("dim", [64, 128])
def test_types(form, dtype, dim):
    """Single tokens, a few, a chunk; a page that ends inside a block."""
    say("types", form, dtype, dim)
    compare(Window([0, 5, 100, 777], [1, 1, 1, 1], 16, 4, 4, dim, form, dtype, 1), tell="tokens")
    compare(Window([0, 90, 3], [70, 33, 200], 32, 2, 2, dim, form, dtype, 2), per_token=True, tell="chunks")
    compare(Window([0, 90, 3], [5, 3, 1], 32, 2, 3, dim, form, dtype, 3), norm=False, tell="few")


@pytest.mark.parametrize("past", [0, 1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 255, 1000, 4095, 4096, 4097])
@pytest.mark.parametrize("dim", [64, 128])
def test_lengths_of_one_token(past, dim):
    say("length", past, dim)
    compare(Window([past], [1], 64, 2, 1, dim, "e4m3", "bf16", past), tell="one head")
    compare(Window([past] * 3, [1] * 3, 16, 6, 5, dim, "int8", "fp16", past), norm=False, per_token=True, tell="three pairs")


@pytest.mark.parametrize("add", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 191, 192, 193, 300])
def test_prompts(add):
    """Rows about the tiles' edges, with and without tokens before them."""
    say("prompt", add)
    compare(Window([0], [add], 16, 2, 1, 64, "e4m3", "fp16", add), tell="empty before")
    compare(Window([77, 0, 1], [add, 1, add // 2 + 1], 128, 4, 1, 128, "int8", "bf16", add), per_token=True, tell="some before")


@pytest.mark.parametrize("group", [1, 2, 3, 7, 8, 16, 17, 65, 128])
def test_groups(group):
    """Query rows that share a pair: parts of a tile up to more than two."""
    say("group", group)
    compare(Window([40, 300], [1, 1], 32, 2, group, 64, "e4m3", "bf16", group), tell="tokens")
    compare(Window([40, 3], [1, 7], 32, 2, group, 128, "e4m3", "bf16", group), norm=False, tell="few")


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("heads", [2, 8, 10])
def test_pages_and_heads(page, heads):
    say("pages", page, heads)
    compare(Window([page - 1, page, 3 * page + 1], [1, 2, page + 1], page, heads, 2, 64, "int8", "bf16", page + heads))


@pytest.mark.parametrize("dim", [64, 128])
def test_work_shared_by_many(dim):
    """Few rows over long contexts (pieces joined, in groups too), and tiles in parts."""
    say("shared work", dim)
    compare(Window([30000], [1], 128, 2, 2, dim, "e4m3", "bf16", 1), tell="one request")
    compare(Window([131000], [1], 128, 2, 1, dim, "int8", "fp16", 2), norm=False, tell="hundreds of pieces")
    compare(Window([20000, 3, 9000], [1, 1, 3], 64, 4, 4, dim, "e4m3", "fp16", 3), tell="uneven")
    compare(Window([6000, 100], [130, 65], 64, 2, 1, dim, "e4m3", "bf16", 4), tell="parts")
    compare(Window([9000], [20], 32, 2, 4, dim, "int8", "bf16", 5), per_token=True, tell="few tiles, many parts")


@pytest.mark.parametrize("requests", [64, 65, 200, 1023, 1025, 2000])
def test_many_requests(requests):
    say("requests", requests)
    past = [(7 * i) % 90 for i in range(requests)]
    compare(Window(past, [1] * requests, 16, 2, 2, 64, "e4m3", "bf16", requests), tell="tokens")
    add = [(3 * i) % 7 if i % 11 else 40 for i in range(requests)]
    compare(Window(past, add, 32, 2, 1, 64, "int8", "fp16", requests), per_token=True, tell="mixed")


@pytest.mark.parametrize("form,most", [("e4m3", 22), ("int8", 29)])
@pytest.mark.parametrize("apart", [0, 1, 12, 22, 29, 33, 60])
@pytest.mark.parametrize("add", [1, 70])
def test_heads_whose_scales_lie_apart(form, most, apart, add):
    """The smaller head's numbers, as exact as the bound says: all bits up to `most`, none far below."""
    say("apart", form, apart, add)
    w = Window([200, 50], [add, 1], 16, 4, 2, 64, form, "fp16", apart)
    w.exps[:, 1::2, 1] -= apart
    _, _, _, out = compare(w, norm=False, gain=1.0)
    w.exps[:, 1::2, 1] += apart
    if apart <= most:
        w.exps[:, 1::2, 1] += 0
        plain = reference(w, lambdas(w, False), None, 1.0, 0.0)[0]
        got = out[..., 64:].double() * 2.0 ** apart
        if apart <= 10:                                     # (an fp16 output holds what lies 2^-10 below)
            assert float((got - plain[..., 64:]).abs().max()) < 0.01 * float(plain.abs().max())
    # page by page in turn
    w.exps[::2, 1::2, 1] -= apart
    w.exps[1::2, 0::2, 1] -= apart
    compare(w, norm=False, gain=1.0)


@pytest.mark.parametrize("dim,add", [(64, 1), (128, 1), (64, 150), (128, 150)])
def test_without_the_second_map_it_is_attention(dim, add):
    """lambda 0: the first halves are what attend makes of even heads."""
    w = Window([300, 20], [add, 1], 32, 4, 3, dim, "e4m3", "bf16", 9)
    tables, cache, step = w.on_gpu()
    zero = torch.zeros(6, device="cuda")
    out = cache.attend_diff(tables, step, w.q, zero, scale=w.scale)
    plain = cache.attend(tables, step, w.q, scale=w.scale).unflatten(1, (2, 2, 3))[:, :, 0].flatten(1, 2)
    room = 2.0 ** -8 * plain.double().abs() * 2 + 2.0 ** -10 * float(plain.abs().max())
    assert bool(((out[..., :dim].double() - plain.double()).abs() <= room).all())


def test_equal_maps_cancel():
    """The same keys, queries and lambda 1: zero within the bound, not NaN, with the norm too."""
    w = Window([500, 10], [1, 80], 16, 2, 2, 64, "e4m3", "fp16", 4)
    w.codes[:, 1, 0], w.exps[:, 1, 0] = w.codes[:, 0, 0], w.exps[:, 0, 0]
    w.q[:, 2:] = w.q[:, :2]
    tables, cache, step = w.on_gpu()
    one = torch.ones(2, device="cuda")
    for weight in (None, torch.ones(128, device="cuda")):
        assert not cache.attend_diff(tables, step, w.q, one, weight=weight, scale=w.scale).any()


def test_what_lies_past_the_tokens_counts_for_nothing():
    """Codes of slots that hold no token yet are NaN, whatever read them; so are other pages'."""
    for add, dim in ((1, 64), (3, 128), (90, 64), (140, 128)):
        w = Window([37, 70, 0], [add, 1, add], 32, 2, 2, dim, "e4m3", "bf16", add)
        used = torch.zeros(w.pages, 32, dtype=torch.bool, device="cuda")
        for row, p, a in zip(w.rows, w.past, w.add):
            for t in range(p + a):
                used[row[t // 32], t % 32] = True
        w.codes[~used[:, None, None, :].expand(-1, 2, 2, -1)] = 0x7F
        ref = w.codes.clone()
        w.codes[w.codes == 0x7F] = 0
        want = reference(w, lambdas(w, False), None, 1.0, 0.0)
        w.codes = ref
        tables, cache, step = w.on_gpu()
        out = cache.attend_diff(tables, step, w.q, lambdas(w, False), scale=w.scale)
        assert bool(((out.double() - want[0]).abs() <= want[2]).all()), add


def test_a_query_that_is_not_finite_spoils_its_own_rows_only():
    for add in (1, 100):
        w = Window([60, 60], [add, 1], 16, 4, 2, 64, "e4m3", "bf16", 3)
        tables, cache, step = w.on_gpu()
        lam, weight = lambdas(w, False), weights(w)
        clean = cache.attend_diff(tables, step, w.q, lam, weight=weight, scale=w.scale)
        q = w.q.clone()
        q[0, 3], q[w.tokens - 1, 4] = float("nan"), float("inf")     # map 1 of pair 0's second head; map 0 of pair 1's first
        out = cache.attend_diff(tables, step, q, lam, weight=weight, scale=w.scale)
        bad = torch.zeros(w.tokens, 4, dtype=torch.bool, device="cuda")
        bad[0, 1] = bad[w.tokens - 1, 2] = True
        assert bool(out[bad].isnan().all()) and torch.equal(out[~bad], clean[~bad])


def test_strides_and_views():
    """Queries out of a wide projection, outputs into a wide tensor, lambda with odd strides."""
    w = Window([300, 9], [2, 70], 16, 4, 2, 64, "e4m3", "bf16", 8)
    tables, cache, step = w.on_gpu()
    lam, weight = lambdas(w, True), weights(w)
    want = cache.attend_diff(tables, step, w.q, lam, weight=weight, scale=w.scale)
    wide = torch.zeros(w.tokens + 5, 3, 8, 64, dtype=torch.bfloat16, device="cuda")
    wide[:w.tokens, 1] = w.q
    into = torch.full((w.tokens + 2, 4, 5, 128), 3.0, dtype=torch.bfloat16, device="cuda")
    turned = torch.zeros(4, w.tokens + 7, device="cuda")
    turned[:, :w.tokens] = lam.t()
    out = cache.attend_diff(tables, step, wide[:, 1], turned.t(), weight=weight, out=into[:, :, 2], scale=w.scale)
    assert torch.equal(out[:w.tokens], want)
    into[:w.tokens, :, 2] = 3.0
    assert bool((into == 3.0).all())
    one = cache.attend_diff(tables, step, w.q, torch.full((1, 1), 0.4, device="cuda").expand(w.tokens, 4), scale=w.scale)
    assert torch.equal(one, cache.attend_diff(tables, step, w.q, torch.full((4,), 0.4, device="cuda"), scale=w.scale))


def test_tokens_without_slots_and_rows_past_the_window():
    cfg = kv_config(4, 64, 3, page=16, heads=2, group=2, dim=64)
    for add, max_new in (([20, 20, 1, 0], 20), ([1, 33, 40, 0], 40)):
        tables, cache = KvTables(cfg), KvCache(cfg)
        n = sum(add)
        step = tables.plan(torch.tensor(add, dtype=torch.int32, device="cuda"), n + 9, max_new=max_new)
        granted = step.granted.tolist()
        assert 0 in granted[:3] and any(granted)
        k, q = (torch.randn(n + 9, h, 64, device="cuda").to(torch.bfloat16) for h in (2, 4))
        cache.append(step, k, k)
        out = torch.full((n + 9, 2, 128), 5.0, device="cuda", dtype=torch.bfloat16)
        lse = torch.full((n + 9, 4), 5.0, device="cuda")
        lam = torch.rand(2, device="cuda")
        cache.attend_diff(tables, step, q, lam, weight=torch.ones(128, device="cuda"), out=out, lse=lse)
        at = 0
        for a, g in zip(add, granted):
            rows = slice(at, at + a)
            if a and not g:
                assert not out[rows].any() and bool((lse[rows] == float("-inf")).all())
            elif a:
                assert bool(out[rows].isfinite().all()) and bool(lse[rows].isfinite().all()) and bool(out[rows].any())
            at += a
        assert bool((out[at:] == 5.0).all()) and bool((lse[at:] == 5.0).all())


def test_more_new_tokens_than_the_bound_says():
    """Rows that no launch makes are NaN, the others right."""
    w = Window([50, 9], [200, 1], 16, 2, 2, 64, "e4m3", "bf16", 8)
    lam = lambdas(w, False)
    right = w.on_gpu()
    want = right[1].attend_diff(right[0], right[2], w.q, lam, scale=w.scale)
    tables, cache, step = w.on_gpu(max_new=1)
    out, lse = torch.zeros_like(want), torch.zeros(w.tokens, 4, device="cuda")
    cache.attend_diff(tables, step, w.q, lam, out=out, lse=lse, scale=w.scale)
    assert bool(out[:200].isnan().all()) and bool(lse[:200].isnan().all())
    assert bool(((out[200:] - want[200:]).abs() <= 2.0 ** -8 * want[200:].abs()).all())


def test_layers_share_a_step_and_a_workspace():
    """Both kinds of attention, other head sizes and forms, one after another on one step."""
    w = Window([9000, 40, 700], [1, 3, 2], 16, 4, 2, 128, "e4m3", "bf16", 5)
    small = Window([9000, 40, 700], [1, 3, 2], 16, 4, 2, 64, "int8", "bf16", 5)
    tables, cache, step = w.on_gpu()
    other = KvCache(kv_config(3, w.row_pages * 16, w.pages, page=16, heads=4, group=2, dim=64, form="int8"))
    other.load(small.codes, small.exps)
    small.rows = w.rows                                              # (the tables are the first layer's)
    for _ in range(3):
        compare(small, on_gpu=(tables, other, step))
        cache.attend(tables, step, w.q)
        compare(w, norm=False, on_gpu=(tables, cache, step))


def test_equal_calls_give_equal_bits():
    """Whoever arrives last at a join."""
    for past, add in (([40000, 100], [1, 1]), ([5000], [140])):
        w = Window(past, add, 32, 2, 2, 64, "e4m3", "bf16", 5)
        tables, cache, step = w.on_gpu()
        lam, weight = lambdas(w, False), weights(w)
        first = cache.attend_diff(tables, step, w.q, lam, weight=weight)
        for _ in range(20):
            assert torch.equal(first, cache.attend_diff(tables, step, w.q, lam, weight=weight))


def test_recorded_into_a_graph():
    """Two layers on one step, replayed with other inputs between eager work."""
    w = Window([3000, 70, 500], [1, 1, 1], 16, 4, 2, 64, "e4m3", "bf16", 6)
    tables, cache, step = w.on_gpu()
    lam, weight = lambdas(w, True), weights(w)
    outs = [torch.empty(3, 4, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    cache.attend_diff(tables, step, w.q, lam, weight=weight, out=outs[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for out in outs:
            cache.attend_diff(tables, step, w.q, lam, weight=weight, out=out)
    for seed in range(4):
        w.q.copy_(torch.randn(w.q.shape, device="cuda"))
        lam.copy_(torch.rand(lam.shape, device="cuda"))
        graph.replay()
        want = cache.attend_diff(tables, step, w.q, lam, weight=weight)
        assert torch.equal(outs[0], want) and torch.equal(outs[1], want)
        torch.cuda.synchronize()


def test_on_a_stream_of_its_own():
    w = Window([300, 70], [1, 90], 16, 4, 2, 64, "e4m3", "bf16", 6)
    tables, cache, step = w.on_gpu()
    lam = lambdas(w, False)
    want = cache.attend_diff(tables, step, w.q, lam)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    for x in (tables, cache, step):
        x.set_stream(stream)
    out = cache.attend_diff(tables, step, w.q, lam)
    stream.synchronize()
    assert torch.equal(out, want)


def test_a_window_of_forks():
    """Forks of prompts, their next tokens, taken back and ended: what the copies of whole requests give."""
    H, G, D, page = 4, 2, 64, 16
    gen = torch.Generator(device="cuda").manual_seed(1)
    lengths, add = [40, 64, 7], [40, 64, 7]
    x = torch.randn(2, 111, H, D, generator=gen, device="cuda").to(torch.bfloat16)
    more = torch.randn(2, 3, H, D, generator=gen, device="cuda").to(torch.bfloat16)
    q = torch.randn(3, H * G, D, generator=gen, device="cuda").to(torch.bfloat16)
    lam = torch.rand(H // 2 * G, generator=gen, device="cuda")
    ints = lambda *z: torch.tensor(z, dtype=torch.int32, device="cuda")          # noqa: E731

    def fill(rows):
        cfg = kv_config(6, 128, 60, page=page, heads=H, group=G, dim=D)
        tables, cache = KvTables(cfg), KvCache(cfg)
        new = [0] * 6
        for r, n in zip(rows, add):
            new[r] = n
        step = tables.plan(ints(*new), 111)
        order = torch.cat([torch.arange(111, device="cuda")[sum(lengths[:j]):sum(lengths[:j + 1])] for j in sorted(range(3), key=lambda j: rows[j])])
        cache.append(step, x[0, order], x[1, order])
        tables.commit(step)
        return tables, cache
    tables, cache = fill([3, 4, 5])
    step = tables.plan(ints(0, 0, 0, 1, 1, 1), 3)
    cache.append(step, *more)
    want = cache.attend_diff(tables, step, q, lam)

    tables, cache = fill([0, 1, 2])
    edit = tables.fork(ints(0, 1, 2), ints(3, 4, 5))
    cache.copy(edit)
    tables.commit(edit)
    step = tables.plan(ints(0, 0, 0, 1, 1, 1), 3)
    cache.append(step, *more)
    assert torch.equal(cache.attend_diff(tables, step, q, lam), want)
    tables.commit(step)
    tables.commit(tables.trim(ints(-1, -1, -1, 40, 64, 7)))         # the new tokens are taken back
    edit = tables.compact()
    cache.copy(edit)
    tables.commit(edit)
    step = tables.plan(ints(0, 0, 0, 1, 1, 1), 3)
    cache.append(step, *more)
    assert torch.equal(cache.attend_diff(tables, step, q, lam), want)
    tables.commit(step)
    tables.commit(tables.trim(ints(0, 0, -1, 0, 0, 0)))
    tables.commit(tables.trim(ints(0, 0, 0, 0, 0, 0)))
    assert tables.counters.tolist()[1:3] == [60, 0] and not tables.owners.any()
