"""Edits whose memory holds anything: commits and copies stay within their buffers."""
import ctypes

import pytest
import torch

from gpu_helpers import say
from paper_2508_01744_amd import KvCache, KvEdit, KvTables, _lib as L, kv_config

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("requests,row_pages,pages", [(3, 2, 9), (70, 5, 1000), (2100, 3, 300)])
@pytest.mark.parametrize("kind", [0, 1, 2, 3, 4])
def test_numbers_that_are_no_places(requests, row_pages, pages, kind):
    """Rows, lengths, moves and counts from -2^31 to 2^31 - 1, and such as are just out of range."""
    say("memory", requests, row_pages, pages, kind)
    cfg = kv_config(requests, row_pages * 16, pages, heads=1, group=1, dim=64)
    tables, cache = KvTables(cfg), KvCache(cfg)
    lib, c = L.lib(), ctypes.byref(tables.cfg)
    edit = KvEdit(cfg, 70000)
    gen = torch.Generator(device="cuda").manual_seed(kind)
    around = torch.tensor([-2 ** 31, -1, 0, 1, requests - 1, requests, row_pages, row_pages + 1, row_pages * 16 + 1, pages - 1,
                           pages, 70000, 70001, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    words = edit.buffer[:edit.nbytes // 4 * 4].view(torch.int32)
    # the tables and the cache between words that have to stay
    wide = [torch.full((b.nbytes + 1024,), 77, dtype=torch.uint8, device="cuda") for b in (tables, cache)]
    inner = []
    for w, b in zip(wide, (tables, cache)):
        at = 256 + -w.data_ptr() % 256
        inner.append(w[at:at + b.nbytes])
        inner[-1].copy_(b.buffer)
    for turn in range(4):
        words.copy_(around[torch.randint(0, len(around), words.shape, generator=gen, device="cuda")])
        edit.counters[7] = kind
        if turn == 3:
            words.fill_(2 ** 31 - 1)
            edit.counters[7] = kind
        before = edit.buffer.clone()
        e = (edit.ptr, edit.nbytes, edit.max_moves)
        assert lib.agft_pages_copy(c, inner[1].data_ptr(), cache.nbytes, *e, None) == 0
        assert lib.agft_pages_commit(c, inner[0].data_ptr(), tables.nbytes, *e, None) == 0
        torch.cuda.synchronize()
        assert torch.equal(edit.buffer, before)
        for w, b in zip(wide, inner):
            start = b.data_ptr() - w.data_ptr()
            assert bool((w[:start] == 77).all()) and bool((w[start + b.numel():] == 77).all())
