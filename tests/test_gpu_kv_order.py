"""Windows, edits and layers' calls in orders that are allowed, on the GPU: results are
those of the same calls on tables and a cache of their own."""
import pytest
import torch

from paper_2508_01744_amd import KvCache, KvStep, KvTables, kv_config

pytestmark = pytest.mark.gpu


def ints(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def test_a_graph_plans_a_step_and_eager_calls_take_it_after_edits():
    """Replays between edits; the last layer's calls and the commit are eager."""
    cfg = kv_config(4, 128, 40, heads=2, group=2, dim=64)
    gen = torch.Generator(device="cuda").manual_seed(3)
    k, v = (torch.randn(2, 2, 64, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2))
    q = torch.randn(2, 4, 64, generator=gen, device="cuda").to(torch.bfloat16)
    add, src, dst, keep = ints(1, 0, 1, 0), ints(0), ints(3), ints(-1, -1, -1, 0)
    sides = []
    for _ in range(2):
        tables, caches = KvTables(cfg), [KvCache(cfg) for _ in range(2)]
        first = tables.plan(ints(40, 0, 7, 0), 47)
        new = torch.randn(47, 2, 64, generator=torch.Generator(device="cuda").manual_seed(4), device="cuda").to(torch.bfloat16)
        for cache in caches:
            cache.append(first, new, new)
        tables.commit(first)
        sides.append((tables, caches, KvStep(cfg, 2, 1)))
    (tables, caches, step), (twin, twins, eager) = sides
    out = torch.empty_like(q)
    twins[0].attend(twin, twin.plan(add, 2, max_new=1, step=eager), q)          # (makes the workspaces)
    tables.plan(add, 2, max_new=1, step=step)
    step.work(caches[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tables.plan(add, 2, max_new=1, step=step)
        caches[0].append(step, k, v)
        caches[0].attend(tables, step, q, out=out)
    for turn in range(4):
        graph.replay()
        caches[1].append(step, k, v)
        got = out.clone(), caches[1].attend(tables, step, q)
        tables.commit(step)
        twin.plan(add, 2, max_new=1, step=eager)
        for cache in twins:
            cache.append(eager, k, v)
        want = [cache.attend(twin, eager, q) for cache in twins]
        twin.commit(eager)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        for t, layers in ((tables, caches), (twin, twins)):
            edit = t.fork(src, dst) if turn % 2 == 0 else t.trim(keep)
            for cache in layers:
                cache.copy(edit)
            t.commit(edit)
        torch.cuda.synchronize()
        assert torch.equal(tables.lengths, twin.lengths) and torch.equal(tables.counters, twin.counters)
