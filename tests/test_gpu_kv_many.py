"""More of the paged cache's attention on the GPU against its 64-bit reference:
chunks over long caches (tiles that several workgroups share), more requests
than a wavefront's lanes and than a workgroup's prefix sums hold, calls in
sequence over one step, and every split of the work around its thresholds.
Bounds as in test_gpu_kv.py."""
import numpy as np
import pytest
import torch

from gpu_helpers import say
from test_gpu_kv import attend_and_compare, fill, ints, make, window_tensors

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim,group,form,dtype", [(64, 4, "e4m3", "bf16"), (128, 3, "int8", "fp16"),
                                                   (256, 5, "e4m3", "fp16"), (128, 8, "int8", "bf16")])
def test_chunk_over_a_long_cache(dim, group, form, dtype):
    """Few tiles of rows over thousands of tokens: parts, some of them empty."""
    rng = np.random.default_rng(dim + group)
    _, tables, cache, node = make(3, 200, 420, 32, 1, group, dim, form)
    step, want = fill(tables, cache, node, rng, [5000, 0, 2050], dtype)
    tables.commit(step)
    node.commit(want)
    for add in ([65 // group + 1, 200 // group, 1], [40, 70, 30]):
        step, want = fill(tables, cache, node, rng, add, dtype)
        say("  worst share of the bound", attend_and_compare(tables, cache, node, step, want, rng, dtype))
        tables.commit(step)
        node.commit(want)


@pytest.mark.parametrize("requests,heads,group,page", [(65, 2, 4, 16), (150, 1, 8, 32), (1100, 1, 2, 16)])
def test_many_requests(requests, heads, group, page):
    """Requests beyond a wavefront's 64 and a workgroup's 1,024, idle and ended
    ones among them, single tokens, drafted ones and chunks."""
    rng = np.random.default_rng(requests)
    _, tables, cache, node = make(requests, 160 // page, requests * 160 // page, page, heads, group, 64, "e4m3")
    first = rng.integers(0, 40, requests)
    step, want = fill(tables, cache, node, rng, first.tolist(), "bf16")
    tables.commit(step)
    node.commit(want)
    for kinds in ((1, 1, 1, 0), (1, 3, 0, -1), (1, 33, 9, 1)):
        add = np.asarray(kinds)[rng.integers(0, 4, requests)]
        add[rng.integers(0, requests)] = 70
        step, want = fill(tables, cache, node, rng, add.tolist(), "bf16")
        say("  worst share of the bound", attend_and_compare(tables, cache, node, step, want, rng, "bf16"))
        tables.commit(step)
        node.commit(want)


@pytest.mark.parametrize("rows", [15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 130, 255, 257])
def test_rows_about_the_tiles_edges(rows):
    """Query rows of a request (one head of its own each) about 16, 64 and 128."""
    rng = np.random.default_rng(rows)
    _, tables, cache, node = make(2, 32, 64, 16, 1, 1, 64, "int8")
    step, want = fill(tables, cache, node, rng, [70, 3], "fp16")
    tables.commit(step)
    node.commit(want)
    step, want = fill(tables, cache, node, rng, [rows, 1], "fp16")
    attend_and_compare(tables, cache, node, step, want, rng, "fp16")


@pytest.mark.parametrize("length", [1, 15, 16, 17, 63, 64, 65, 191, 192, 193, 255, 256, 257, 1023, 1024, 1025, 2047, 2049])
def test_lengths_about_the_units_edges(length):
    """One request whose tokens end about a block, a unit, a workgroup's share."""
    rng = np.random.default_rng(length)
    for dim, heads in ((64, 3), (128, 1), (256, 2)):
        _, tables, cache, node = make(1, 140, 140, 16, heads, 2, dim, "e4m3")
        step, want = fill(tables, cache, node, rng, [length], "bf16")
        if length <= 20:
            attend_and_compare(tables, cache, node, step, want, rng, "bf16")
        tables.commit(step)
        node.commit(want)
        step, want = fill(tables, cache, node, rng, [1], "bf16")
        attend_and_compare(tables, cache, node, step, want, rng, "bf16")


def test_layers_share_a_step():
    """Many calls over one step and one workspace: each gives what it gives alone."""
    rng = np.random.default_rng(21)
    _, tables, cache, node = make(3, 260, 800, 16, 2, 4, 128, "e4m3")
    step, want = fill(tables, cache, node, rng, [4000, 900, 33], "bf16")
    tables.commit(step)
    node.commit(want)
    step, want = fill(tables, cache, node, rng, [1, 40, 3], "bf16")
    qs = [window_tensors(rng, step.max_tokens, 8, 128, torch.bfloat16)[0] for _ in range(4)]
    rows = want["starts"][-1]
    alone = []
    for q in qs:
        alone.append(cache.attend(tables, step, q)[:rows].clone())
        torch.cuda.synchronize()
    for _ in range(3):
        outs = [cache.attend(tables, step, q)[:rows] for q in qs]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(alone, outs))
    # and a smaller launch of the same step's kind between them
    other = tables.plan(ints([1, 1, 1]), 3, max_new=1)
    q = qs[0][:3]
    lone = cache.attend(tables, other, q).clone()
    cache.attend(tables, step, qs[1])
    assert torch.equal(cache.attend(tables, other, q), lone)


def test_out_and_queries_with_strides():
    """Outputs into a view with gaps, queries with heads apart, logarithms beside."""
    rng = np.random.default_rng(30)
    _, tables, cache, node = make(2, 8, 16, 32, 2, 3, 64, "int8")
    step, want = fill(tables, cache, node, rng, [60, 9], "fp16")
    n = step.max_tokens
    q = torch.randn(6, n, 64, device="cuda").half().transpose(0, 1)          # [n][6][64], heads outermost in memory
    packed = cache.attend(tables, step, q.contiguous())
    wide = torch.full((n, 6, 128), 3.0, dtype=torch.float16, device="cuda")
    cache.attend(tables, step, q, out=wide[:, :, 64:])
    assert torch.equal(wide[:69, :, 64:], packed[:69])
    assert (wide[:, :, :64] == 3.0).all() and (wide[69:] == 3.0).all()


@pytest.mark.parametrize("requests", [20, 60])
def test_some_rows_over_little_and_much_work(requests):
    """17 to 64 query rows per request: the split over tokens while that is little
    work in all (20 requests), tiles of rows beyond (60)."""
    rng = np.random.default_rng(requests)
    _, tables, cache, node = make(requests, 26, requests * 26, 128, 1, 8, 64, "e4m3")
    lengths = [2500 + 7 * i for i in range(requests)]
    step, want = fill(tables, cache, node, rng, lengths, "bf16")
    tables.commit(step)
    node.commit(want)
    add = [3 + i % 6 for i in range(requests)]
    units = sum(-(-(n + a) // 64) * -(-8 * a // 16) for n, a in zip(lengths, add))
    assert (units <= 6144) == (requests == 20)
    step, want = fill(tables, cache, node, rng, add, "bf16")
    say("  worst share of the bound", attend_and_compare(tables, cache, node, step, want, rng, "bf16"))
