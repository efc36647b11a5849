"""Python front end of the serving node's paged cache (agft_kv.h, agft_pages.h, agft_diff.h): torch
supplies device memory and streams, the work runs in the HIP kernels behind
libagft.so.

One window of a node with a KvTables `tables` and, per layer, a KvCache `cache`:

    step = tables.plan(add, max_tokens)        # pages and slots of the new tokens
    cache.append(step, k, v)                   # per layer
    out = cache.attend(tables, step, q)        # per layer (or attend_diff)
    tables.commit(step)                        # the new lengths become the tables'

and between windows the tables can be edited (agft_pages.h):

    edit = tables.fork(src, dst)               # or trim(keep), or compact()
    cache.copy(edit)                           # per layer
    tables.commit(edit)

Calls enqueue on the stream given to the object, or else on the stream that is
current when they are called; nothing here waits for the GPU except load().
There is no backward pass: tensors that ask for a gradient are refused.
Launches go to the calling thread's current device, which has to be the object's.
Tensors of another stream are the caller's to order, as for any torch call.
Windows and edits are planned one at a time, each committed before the next is
planned: plans write into the tables' rows and ring, where a later one writes over
an earlier one.  So what was planned before the latest plan is not committed any
more (plan it again), and nor do layers take an edit or store tokens of a window
then, unless that had been committed; steps and edits of tables that were edited,
loaded or reset since are refused too, and those of other tables.  (Of two windows
the older one's step still attends, to the pages that the rows name now.)  A graph's replays are not
watched: a step that a graph plans is taken as the caller says it is.
"""
import contextlib
import ctypes
import math

import torch

from . import _lib as L

FORMS = {"e4m3": L.AGFT_KV_E4M3, "int8": L.AGFT_KV_INT8}
TYPES = {torch.bfloat16: L.AGFT_KV_BF16, torch.float16: L.AGFT_KV_FP16, torch.float32: L.AGFT_KV_FP32}


def kv_config(requests, row_tokens, pages, page=16, heads=8, group=4, dim=128, form="e4m3"):
    """The agft_kv_config of a node: rows of the block table, tokens a request
    can hold, pages of the pool, tokens of a page, key/value heads, query heads
    per key/value head, numbers of a head, and how the cache holds them
    ("e4m3" or "int8").  No device work."""
    if form not in FORMS:
        raise ValueError(f"form must be one of {sorted(FORMS)}, not {form!r}")
    page = int(page)
    if page < 1:
        raise ValueError("a page holds at least one token")
    return L.agft_kv_config(int(requests), -(-int(row_tokens) // page), int(pages), page, int(heads), int(group),
                            int(dim), FORMS[form])


try:
    _current_raw_stream = torch._C._cuda_getCurrentRawStream
except AttributeError:
    def _current_raw_stream(index):
        return torch.cuda.current_stream(index).cuda_stream

try:
    _current_device = torch._C._cuda_getDevice
except AttributeError:
    _current_device = torch.cuda.current_device

_recording = torch.cuda.is_current_stream_capturing


_one = {}       # devices and configurations' tuples, one object each: compared at every call


def _device(device):
    device = torch.device(device)
    if device.type == "cuda" and device.index is None:
        device = torch.device("cuda", torch.cuda.current_device())
    return _one.setdefault(device, device)


class _OnStream:
    """What the front ends share: a configuration, a device, a stream.  Tables,
    steps and caches that meet in a call have to have one configuration (a layer's
    dim and form are its own)."""

    def _init(self, cfg, device, stream):
        # (a copy: sizes and layouts follow from it)
        self.cfg, self.device = type(cfg).from_buffer_copy(cfg), _device(device)
        self._index = self.device.index
        self.set_stream(stream)
        self._cfg = ctypes.byref(self.cfg)
        self._lib = L.lib()
        # where the parts of tables and steps lie; layers may differ in dim and form
        shape = cfg.requests, cfg.row_pages, cfg.pages, cfg.page, cfg.heads, cfg.group
        self._shape = _one.setdefault(shape, shape)

    def _fits(self, other, what):
        """Refuse tables and steps of other devices or configurations, and steps without a plan."""
        if other.device is not self.device and other.device != self.device:
            raise ValueError(f"{what} on {other.device}, not {self.device}")
        if other._shape is not self._shape:
            raise ValueError(f"{what} of another configuration: (requests, row_pages, pages, page, heads, group) "
                             f"{other._shape}, not {self._shape}")
        if not other.planned:
            raise ValueError(f"the {what} has not been planned: its memory holds nothing yet")

    def _fits_step(self, step):
        """And steps whose slots and lengths are of tables that were edited, loaded or reset since."""
        self._fits(step, "step")
        if step._number <= step._of._void and not step._recorded:
            raise ValueError("the tables have been edited, loaded or reset since the step was planned")

    def _fits_window(self, tables, step):
        """What attends: the step, and its tables as no edit's plan has written into them."""
        self._fits_step(step)
        self._fits(tables, "tables")
        if step._recorded:
            return
        if step._of is not tables:
            raise ValueError("the step was planned from other tables")
        if step._number < tables._edit_number and not step._done:
            raise ValueError("an edit has been planned since the step, which was not committed: its rows may be the "
                             "edit's by now")

    def set_stream(self, stream):
        """Enqueue on `stream` from now on (None: on the stream current at each call)."""
        if stream is not None and stream.device != self.device:
            raise ValueError(f"a stream of {stream.device} for work on {self.device}")
        self.stream = stream

    def _s(self):
        if _current_device() != self._index:
            raise ValueError(f"work on {self.device} while the current device is {_current_device()}: launches go to "
                             "the current device")
        # (the raw handle: a window's calls are short enough for the Stream object's microseconds to count)
        return _current_raw_stream(self._index) if self.stream is None else self.stream.cuda_stream

    @contextlib.contextmanager
    def _settled(self):
        """Set-up work on the object's stream: after what the caller's stream
        holds, and done when it ends, so that any stream may go on from there."""
        torch.cuda.current_stream(self.device).synchronize()
        with torch.cuda.stream(self.stream) if self.stream is not None else contextlib.nullcontext():
            yield
            torch.cuda.current_stream(self.device).synchronize()

    def _empty(self, *shape, dtype):
        """Memory that belongs to the stream which the work on it is enqueued on."""
        if self.stream is None:
            return torch.empty(*shape, dtype=dtype, device=self.device)
        with torch.cuda.stream(self.stream):
            return torch.empty(*shape, dtype=dtype, device=self.device)

    def _buffer(self, nbytes, what):
        if nbytes == 0:
            raise ValueError(f"invalid {what} configuration")
        return self._empty(nbytes, dtype=torch.uint8)

    def _ints(self, t, shape, what):
        if t.get_device() != self._index or t.dtype != torch.int32 or t.shape != shape or not t.is_contiguous():
            raise ValueError(f"{what} must be a contiguous int32 tensor {list(shape)} on {self.device}")


def _view(buf, ptr, dtype, shape):
    off = ptr - buf.data_ptr()
    count = math.prod(shape) * dtype.itemsize
    return buf[off:off + count].view(dtype).view(shape)


class KvStep(_OnStream):
    """A window that KvTables.plan writes, on the GPU (`planned` once it has):

    counters [8]  after the window: ring's head, free pages; the window's
                  tokens, requests refused, pages taken, pages given back
    lengths [R]   after the window, granted [R] new tokens that got slots
    starts [R+1]  first row of each request in the window's tensors
    slots [max_tokens] int64, -1 where nothing is stored
    """

    def __init__(self, cfg, max_tokens, max_new=None, device="cuda", stream=None):
        self._init(cfg, device, stream)
        self.max_tokens = int(max_tokens)
        if not 1 <= self.max_tokens <= 1 << 30:
            raise ValueError("max_tokens must be in 1..2^30")
        self.set_max_new(max_new)
        self.nbytes = self._lib.agft_kv_step_bytes(self._cfg, self.max_tokens)
        self.buffer = self._buffer(self.nbytes, "cache")
        self.ptr = self.buffer.data_ptr()
        v = L.agft_kv_step_view()
        L.check("agft_kv_step_at", self._lib.agft_kv_step_at(self._cfg, self.max_tokens, self.ptr, self.nbytes,
                                                             ctypes.byref(v)))
        R = cfg.requests
        self.counters = _view(self.buffer, v.counters, torch.int32, (8,))
        self.lengths = _view(self.buffer, v.lengths, torch.int32, (R,))
        self.granted = _view(self.buffer, v.granted, torch.int32, (R,))
        self.starts = _view(self.buffer, v.starts, torch.int32, (R + 1,))
        self.slots = _view(self.buffer, v.slots, torch.int64, (self.max_tokens,))
        self._works, self._work_dim = [], 0
        self._diff_works, self._diff_dim = [], 0
        # the tables that it was planned from, by which of their plans, and whether that was committed (of a step
        # that a graph plans all that is as the caller says: nobody here sees its replays)
        self.planned, self._of, self._number, self._done, self._recorded = False, None, 0, False, False

    def set_max_new(self, max_new):
        """No request brings more new tokens than this (None: max_tokens); rows
        of requests that do may come back from attend as NaN."""
        self.max_new = self.max_tokens if max_new is None else int(max_new)
        if not 1 <= self.max_new <= self.max_tokens:
            raise ValueError("max_new must be in 1..max_tokens")

    def work(self, owner=None):
        """The attention's workspace, shared by the layers, which run one after
        another; made for the stream of `owner` when it is first asked for, and
        again for a layer of larger heads than those before (the older ones stay: a
        recorded graph may hold them)."""
        owner = owner or self
        if owner.cfg.dim > self._work_dim:
            self._works.append(owner._buffer(self._lib.agft_kv_attend_bytes(owner._cfg, self.max_tokens), "cache"))
            self._work_dim = owner.cfg.dim
        return self._works[-1]

    def diff_work(self, owner):
        """The same of the differential attention."""
        if owner.cfg.dim > self._diff_dim:
            self._diff_works.append(owner._buffer(self._lib.agft_diff_attend_bytes(owner._cfg, self.max_tokens), "cache"))
            self._diff_dim = owner.cfg.dim
        return self._diff_works[-1]


class KvEdit(_OnStream):
    """An edit that KvTables.fork, trim or compact writes, on the GPU (`planned` once one has):

    counters [8]         after the edit: ring's head, free pages, owners beyond the first of all pages;
                         requests refused, pages taken, pages given back, entries of moves, kind
    lengths [R]          after the edit
    granted [max_moves]  of a fork: tokens that each one got
    moves [max_moves][2] pages to copy, from and to; -1 where there is none
    """

    def __init__(self, cfg, max_moves, device="cuda", stream=None):
        self._init(cfg, device, stream)
        self.max_moves = int(max_moves)
        if not 1 <= self.max_moves <= 1 << 27:
            raise ValueError("max_moves must be in 1..2^27")
        self.nbytes = self._lib.agft_pages_edit_bytes(self._cfg, self.max_moves)
        self.buffer = self._buffer(self.nbytes, "cache")
        self.ptr = self.buffer.data_ptr()
        v = L.agft_pages_view()
        L.check("agft_pages_edit_at", self._lib.agft_pages_edit_at(self._cfg, self.max_moves, self.ptr, self.nbytes,
                                                                   ctypes.byref(v)))
        self.counters = _view(self.buffer, v.counters, torch.int32, (8,))
        self.lengths = _view(self.buffer, v.lengths, torch.int32, (cfg.requests,))
        self.granted = _view(self.buffer, v.granted, torch.int32, (self.max_moves,))
        self.moves = _view(self.buffer, v.moves, torch.int32, (self.max_moves, 2))
        # the tables that it was planned from, by which of their plans, after how many of their changes, and whether
        # it is one of them
        self.planned, self._of, self._number, self._when, self._done = False, None, 0, -1, False


class KvTables(_OnStream):
    """Block tables, lengths and the ring of free pages of a node's requests:
    counters [8], lengths [R], table [R][row_pages], ring [pages], owners [pages]
    beyond a page's first (int32).  While a page has several owners, counters[2] is
    not 0, and requests end by trim: a plan refuses to end them.  Where owners were not
    counted (load), counters[3] is 1, and trims are refused too."""
    planned = True      # (as a step's: their memory holds something from the start)

    def __init__(self, cfg, device="cuda", stream=None):
        self._init(cfg, device, stream)
        self.nbytes = self._lib.agft_kv_tables_bytes(self._cfg)
        self.buffer = self._buffer(self.nbytes, "cache")
        self.ptr = self.buffer.data_ptr()
        v = L.agft_kv_tables_view()
        L.check("agft_kv_tables_at", self._lib.agft_kv_tables_at(self._cfg, self.ptr, self.nbytes, ctypes.byref(v)))
        self.counters = _view(self.buffer, v.counters, torch.int32, (8,))
        self.lengths = _view(self.buffer, v.lengths, torch.int32, (cfg.requests,))
        self.table = _view(self.buffer, v.table, torch.int32, (cfg.requests, cfg.row_pages))
        self.ring = _view(self.buffer, v.ring, torch.int32, (cfg.pages,))
        owners = ctypes.c_void_p()
        L.check("agft_pages_owners_at", self._lib.agft_pages_owners_at(self._cfg, self.ptr, self.nbytes,
                                                                       ctypes.byref(owners)))
        self.owners = _view(self.buffer, owners.value, torch.int32, (cfg.pages,))
        # Changes of the tables; the latest plan's number, the latest windows' and edits' ones, and the last one that
        # an edit, a load or a reset has left behind: plans hold for the tables that they were made from.
        self._changes = self._number = self._step_number = self._edit_number = self._void = 0
        self._token = object()      # what layers know them by
        self.reset()

    def reset(self):
        """No request holds a token, every page is free."""
        L.check("agft_kv_reset", self._lib.agft_kv_reset(self._cfg, self.ptr, self.nbytes, self._s()))
        self._changes += 1
        self._void = self._number
        self._partly = False

    def load(self, lengths, table, free, shared=False):
        """Take over the tables of a running node: lengths [R], table
        [R][row_pages] and the free pages in the order of their use (int32), which
        no request holds and of which none is named twice.
        shared: requests may have pages in common, whose owners are counted.  While
        one of them is a request's last, filled in part, windows that bring that
        request tokens are refused, and plans wait for the GPU to see whether they do.
        Without it pages in common stay whole: no request ends or is trimmed (both
        count as refused), and such a page that is filled in part is refused.
        Set-up: checks the values, which waits for the GPU."""
        cfg = self.cfg
        self._ints(lengths, (cfg.requests,), "lengths")
        self._ints(table, (cfg.requests, cfg.row_pages), "table")
        if free.dim() != 1 or free.numel() > cfg.pages:
            raise ValueError("free must list at most the pool's pages")
        self._ints(free, (free.numel(),), "free")
        bad = [((t < 0) | (t >= top)).any() for t, top in ((lengths, cfg.row_pages * cfg.page + 1), (table, cfg.pages),
                                                           (free, cfg.pages))]
        for wrong, what in zip(torch.stack(bad).tolist(), ("lengths", "table", "free")):
            if wrong:
                raise ValueError(f"{what} out of range")
        used = torch.arange(cfg.row_pages, device=table.device) < ((lengths + (cfg.page - 1)) // cfg.page)[:, None]
        holders = torch.bincount(table[used], minlength=cfg.pages)
        listed = torch.bincount(free, minlength=cfg.pages)
        twice, held = torch.stack([(listed > 1).any(), ((listed > 0) & (holders > 0)).any()]).tolist()
        if twice:
            raise ValueError("free lists a page twice")
        if held:
            raise ValueError("free lists a page that a request holds")
        # (of requests whose last page is filled in part: whether others hold that page)
        last = table.gather(1, (lengths // cfg.page).clamp(max=cfg.row_pages - 1).long()[:, None])[:, 0].long()
        common, partly = torch.stack([(holders > 1).any(), ((lengths % cfg.page != 0) & (holders[last] > 1)).any()]).tolist()
        if partly and not shared:
            raise ValueError("a page that its request fills in part is another's too: without shared both would write there")
        counters = torch.tensor([0, free.numel(), 0, int(common and not shared), 0, 0, 0, 0], dtype=torch.int32)
        owners = None
        if shared:
            owners = (holders - 1).clamp_(min=0)
            counters[2] = owners.sum()
        with self._settled():
            self.owners.zero_() if owners is None else self.owners.copy_(owners)
            self.lengths.copy_(lengths)
            self.table.copy_(table)
            self.ring.zero_()
            self.ring[:free.numel()].copy_(free)
            self.counters.copy_(counters)
        self._partly = partly
        self._changes += 1
        self._void = self._number

    def plan(self, add, max_tokens, max_new=None, step=None):
        """Plan a window: add [R] int32 new tokens per request (0: none, < 0: it
        ends), at most max_tokens in all and max_new per request (bounds the
        host knows).  step: a KvStep of the same max_tokens to write again."""
        self._ints(add, (self.cfg.requests,), "add")
        if step is None:
            step = KvStep(self.cfg, max_tokens, max_new, self.device, self.stream)
        else:
            if step.device != self.device or step._shape is not self._shape:
                self._fits(step, "step")
            if step.max_tokens != max_tokens:
                raise ValueError(f"step is for {step.max_tokens} tokens, not {max_tokens}")
            step.set_max_new(max_new)
        if self._partly:
            self._look_for_writes(add)
        code = self._lib.agft_kv_plan(self._cfg, self.ptr, self.nbytes, add.data_ptr(), step.ptr, step.nbytes,
                                      step.max_tokens, self._s())
        if code != L.AGFT_OK:
            L.check("agft_kv_plan", code)
        if self.device.type == "cuda" and _recording():
            step._recorded = True
        else:
            self._number += 1
            self._step_number = self._number
        step.planned, step._of, step._number, step._done = True, self, self._number, False
        return step

    def _look_for_writes(self, add):
        """Tables that were loaded with a partly filled page in common: whether this
        window would write into one, until there is none any more."""
        if self.device.type == "cuda" and _recording():
            raise ValueError("tables with a partly filled page in common: windows can be recorded once it has one owner")
        with self._settled():
            inside = self.lengths % self.cfg.page
            last = self.table.gather(1, (self.lengths // self.cfg.page).clamp(max=self.cfg.row_pages - 1).long()[:, None])
            partly = (inside != 0) & (self.owners[last[:, 0].long()] > 0)
            partly, meets = torch.stack([partly.any(), (partly & (add > 0)).any()]).tolist()
        if meets:
            raise ValueError("new tokens of a request whose last page, filled in part, is another's too: end one of them")
        self._partly = partly

    def commit(self, step):
        """The planned window's lengths and free pages, or the planned edit, become the tables'."""
        if isinstance(step, KvEdit):
            return self._commit_edit(step)
        self._fits_step(step)
        if step._of is not self and not step._recorded:
            raise ValueError("the step was planned from other tables")
        if step._number != self._number and not step._recorded:
            raise ValueError("another window or an edit has been planned since the step: it may have written over its pages")
        L.check("agft_kv_commit", self._lib.agft_kv_commit(self._cfg, self.ptr, self.nbytes, step.ptr, step.nbytes,
                                                           step.max_tokens, self._s()))
        self._changes += 1
        step._done = True

    def _edit(self, name, edit, moves, *args):
        """Plan an edit with room for `moves` moves."""
        if edit is None:
            edit = KvEdit(self.cfg, moves, self.device, self.stream)
        elif edit._shape is not self._shape or edit.device != self.device:
            raise ValueError("edit of another device or configuration")
        code = getattr(self._lib, name)(self._cfg, self.ptr, self.nbytes, *args, edit.ptr, edit.nbytes,
                                                        edit.max_moves, self._s())
        if code != L.AGFT_OK:
            L.check(name, code)
        self._number += 1
        self._edit_number = self._number
        edit.planned, edit._of, edit._number, edit._when, edit._done = True, self, self._number, self._changes, False
        return edit

    def fork(self, src, dst, tokens=None, edit=None):
        """Plan forks: request dst[j] gets the first tokens[j] (all if None) tokens
        of request src[j]; int32 [n], n in 1..65536.  Whole pages are shared, a
        partly filled last one is copied (KvCache.copy).  dst[j] holds nothing and
        is named once; edit.granted[j] is 0 where that is not so, or no page is
        free.  edit: a KvEdit of max_moves n to write again."""
        shape = src.shape
        n = shape[0] if len(shape) == 1 else 0
        if not 1 <= n <= 65536:
            raise ValueError("src must name 1 to 65536 requests")
        self._ints(src, shape, "src")
        self._ints(dst, shape, "dst")
        if tokens is not None:
            self._ints(tokens, shape, "tokens")
        if edit is not None and edit.max_moves != n:
            raise ValueError(f"edit is for {edit.max_moves} moves, not {n}")
        return self._edit("agft_pages_fork", edit, n, src.data_ptr(), dst.data_ptr(), None if tokens is None else tokens.data_ptr(), n)

    def trim(self, keep, edit=None):
        """Plan that request i keeps its first keep[i] tokens (int32 [R]; 0 ends it,
        a negative number or one not below its length keeps all).  Pages without an
        owner are free after the commit.  A request that would end inside a page
        with other owners stays as it is and counts as refused.  No pages to copy."""
        self._ints(keep, (self.cfg.requests,), "keep")
        return self._edit("agft_pages_trim", edit, 1, keep.data_ptr())

    def compact(self, edit=None):
        """Plan that the held pages go to the pool's lower end: afterwards the free
        ones are its last, in ascending order.  The pages that move have to be
        copied in every layer (KvCache.copy).  edit: one of max_moves
        max(1, pages // 2) to write again."""
        moves = max(1, self.cfg.pages // 2)
        if edit is not None and edit.max_moves != moves:
            raise ValueError(f"edit is for {edit.max_moves} moves, not {moves}")
        return self._edit("agft_pages_compact", edit, moves)

    def _commit_edit(self, edit):
        self._fits(edit, "edit")
        if edit._of is not self or edit._when != self._changes or edit._done:
            raise ValueError("the tables have changed since the edit was planned, or it is not theirs")
        if edit._number != self._number:
            raise ValueError("a window or another edit has been planned since the edit: it may have written over its "
                             "rows and free pages")
        L.check("agft_pages_commit", self._lib.agft_pages_commit(self._cfg, self.ptr, self.nbytes, edit.ptr, edit.nbytes,
                                                                 edit.max_moves, self._s()))
        self._changes += 1
        self._void = self._number
        edit._when, edit._done = self._changes, True


class KvCache(_OnStream):
    """One layer's pages: 8-bit codes and an exponent per page, head and side."""

    def __init__(self, cfg, device="cuda", stream=None):
        self._init(cfg, device, stream)
        # what calls tell the library of their tensors (a front end is not thread-safe, like a Tuner)
        self._d0, self._d1 = L.agft_kv_dense(), L.agft_kv_dense()
        self._b0, self._b1 = ctypes.byref(self._d0), ctypes.byref(self._d1)
        self._diff = L.agft_diff_args()
        self._bdiff = ctypes.byref(self._diff)
        # the latest window appended and edit copied here, by their plans' numbers and their tables: what an edit's
        # plan found in its pages is there from the windows before it until the copy, and from the copy on
        self._appended, self._appended_of, self._copied, self._copied_of = 0, None, 0, None
        self.nbytes = self._lib.agft_kv_cache_bytes(self._cfg)
        self.buffer = self._buffer(self.nbytes, "cache")
        self.ptr = self.buffer.data_ptr()
        count = cfg.pages * cfg.heads * 2
        # codes by blocks (agft_kv.h), exponents behind them
        self.codes = self.buffer[:count * cfg.page * cfg.dim].view(cfg.pages, cfg.heads, 2, cfg.page * cfg.dim)
        at = -(-count * cfg.page * cfg.dim // 256) * 256
        self.exps = self.buffer[at:at + 4 * count].view(torch.int32).view(cfg.pages, cfg.heads, 2)

    def load(self, codes, exps):
        """Take over codes uint8 [pages][heads][2][page][dim] (keys, values) and
        exponents int32 [pages][heads][2] in -126..126.  Set-up: checks the
        exponents, waits for the GPU."""
        c = self.cfg
        if codes.dtype != torch.uint8 or tuple(codes.shape) != (c.pages, c.heads, 2, c.page, c.dim):
            raise ValueError("codes must be uint8 [pages][heads][2][page][dim]")
        if exps.dtype != torch.int32 or tuple(exps.shape) != (c.pages, c.heads, 2):
            raise ValueError("exps must be int32 [pages][heads][2]")
        self._dev(codes), self._dev(exps)
        if bool(((exps < -126) | (exps > 126)).any()):
            raise ValueError("exponents out of range: -126..126")
        with self._settled():
            self.exps.copy_(exps)
            part = max(1, (1 << 28) // (c.heads * 2 * c.page * c.dim))
            for p in range(0, c.pages, part):
                q = min(c.pages, p + part)
                lead = (q - p, c.heads, c.page // 16)
                k = codes[p:q, :, 0].reshape(*lead, 16, c.dim // 64, 4, 16)
                self.codes[p:q, :, 0] = k.permute(0, 1, 2, 4, 5, 3, 6).reshape(q - p, c.heads, -1)
                v = codes[p:q, :, 1].reshape(*lead, 4, 4, c.dim // 64, 4, 16)
                self.codes[p:q, :, 1] = v.permute(0, 1, 2, 5, 3, 7, 6, 4).reshape(q - p, c.heads, -1)

    def _dev(self, t):
        if t.device != self.device:
            raise ValueError(f"expected a tensor on {self.device}")

    def _dense(self, d, t, heads, rows, what, types=TYPES, dim=None):
        """Fill the agft_kv_dense d from a [tokens][heads][dim] tensor of at least `rows` tokens."""
        if dim is None:
            dim = self.cfg.dim
        try:
            n, h, last = t.shape
            token, head, one = t.stride()
            kind = types[t.dtype]
        except (ValueError, KeyError):
            n = h = last = one = -1
        if n < rows or h != heads or last != dim or one != 1 or t.get_device() != self._index:
            raise ValueError(f"{what} must be [{rows} or more][{heads}][{dim}] on {self.device}, "
                             f"{' or '.join(str(d) for d in types)}, with contiguous numbers of a head")
        if t.requires_grad and torch.is_grad_enabled():
            raise ValueError(f"{what} asks for a gradient, and these calls have none: detach it, or call under "
                             "torch.no_grad()")
        ptr = t.data_ptr()
        per = 7 if kind != L.AGFT_KV_FP32 else 3
        if ptr & 15 or token & per or head & per:
            raise ValueError(f"{what}: rows must start at multiples of 16 bytes")
        d.data, d.token_stride, d.head_stride, d.type = ptr, token, head, kind

    def append(self, step, k, v):
        """Store the window's keys and values, [max_tokens][heads][dim] each
        (bf16, fp16 or fp32), rows as in step.starts."""
        H, n = self.cfg.heads, step.max_tokens
        self._fits_step(step)
        if step._number < step._of._step_number and not (step._done or step._recorded):
            raise ValueError("another window has been planned since the step, which was not committed: its slots may be "
                             "that one's by now")
        if self._copied > step._number and self._copied_of is step._of._token and not step._recorded:
            raise ValueError("the pages of a later edit have been copied in this layer: append a window before that, or "
                             "plan it after the edit's commit")
        if k.dtype != v.dtype:
            raise ValueError("k and v must have one type")
        self._dense(self._d0, k, H, n, "k")
        self._dense(self._d1, v, H, n, "v")
        code = self._lib.agft_kv_append(self._cfg, self.ptr, self.nbytes, step.ptr, step.nbytes, n, self._b0, self._b1,
                                        self._s())
        if code != L.AGFT_OK:
            L.check("agft_kv_append", code)
        if not step._recorded:
            self._appended, self._appended_of = step._number, step._of._token

    def attend(self, tables, step, q, out=None, lse=None, scale=None):
        """softmax(scale q K^T) V of the window's tokens over their requests'
        tokens up to themselves.  q, out [max_tokens][heads * group][dim], bf16
        or fp16 (out is allocated if None; rows past the window's tokens stay as
        they are, in a fresh one whatever its memory held); lse float32
        [max_tokens][heads * group] or None receives the logarithms of the sums;
        scale: 1 / sqrt(dim) if None."""
        c, n = self.cfg, step.max_tokens
        hq = c.heads * c.group
        self._fits_window(tables, step)
        if out is None:
            out = self._empty(n, hq, c.dim, dtype=q.dtype)
        elif out.dtype != q.dtype:
            raise ValueError("q and out must have one type")
        self._dense(self._d0, q, hq, n, "q", HALVES)
        self._dense(self._d1, out, hq, n, "out", HALVES)
        if lse is not None and (lse.device != self.device or lse.dtype != torch.float32 or
                                lse.shape != (n, hq) or not lse.is_contiguous()):
            raise ValueError(f"lse must be a contiguous float32 tensor [{n}][{hq}] on {self.device}")
        work = step.work(self)
        code = self._lib.agft_kv_attend(self._cfg, self.ptr, self.nbytes, tables.ptr, tables.nbytes, step.ptr,
                                        step.nbytes, n, step.max_new, self._b0, self._b1,
                                        None if lse is None else lse.data_ptr(),
                                        1.0 / math.sqrt(c.dim) if scale is None else float(scale), work.data_ptr(),
                                        work.numel(), self._s())
        if code != L.AGFT_OK:
            L.check("agft_kv_attend", code)
        return out

    def attend_diff(self, tables, step, q, lam, weight=None, gain=1.0, eps=1e-5, out=None, lse=None, scale=None):
        """Differential attention (agft_diff.h): heads 2 p and 2 p + 1 are a pair,
        y = (softmax(scale q_0 K_0^T) - lam softmax(scale q_1 K_1^T)) [V_0 V_1], and out
        is gain y, or with a weight (float32 [2 dim]) gain weight y / sqrt(mean(y^2) +
        eps).  q [max_tokens][heads * group][dim], as for attend (q_0 and q_1 lie group
        heads apart: a projection that puts them side by side needs its rows permuted
        when group > 1); lam float32
        [heads / 2 * group], or [max_tokens][heads / 2 * group] with any strides; out
        [max_tokens][heads / 2 * group][2 * dim]; lse, scale and rows past the window's
        tokens as in attend."""
        c, n = self.cfg, step.max_tokens
        hq, ho = c.heads * c.group, c.heads // 2 * c.group
        self._fits_window(tables, step)
        if c.heads % 2 or c.dim not in (64, 128):
            raise ValueError(f"differential attention is of pairs of heads of 64 or 128 numbers, not {c.heads} of {c.dim}")
        if out is None:
            out = self._empty(n, ho, 2 * c.dim, dtype=q.dtype)
        elif out.dtype != q.dtype:
            raise ValueError("q and out must have one type")
        self._dense(self._d0, q, hq, n, "q", HALVES)
        self._dense(self._d1, out, ho, n, "out", HALVES, 2 * c.dim)
        if lse is not None and (lse.device != self.device or lse.dtype != torch.float32 or
                                lse.shape != (n, hq) or not lse.is_contiguous()):
            raise ValueError(f"lse must be a contiguous float32 tensor [{n}][{hq}] on {self.device}")
        shape = lam.shape
        if shape == (ho,):
            token, (head,) = 0, lam.stride()
        elif len(shape) == 2 and shape[1] == ho and shape[0] >= n:
            token, head = lam.stride()
        else:
            token = None
        if token is None or lam.dtype != torch.float32 or lam.get_device() != self._index:
            raise ValueError(f"lam must be float32 [{ho}] or [{n} or more][{ho}] on {self.device}")
        at = None
        if weight is not None:
            at = weight.data_ptr()
            if weight.shape != (2 * c.dim,) or weight.dtype != torch.float32 or at & 15 or weight.get_device() != self._index \
                    or not weight.is_contiguous():
                raise ValueError(f"weight must be a contiguous float32 tensor [{2 * c.dim}] on {self.device}, from a multiple "
                                 "of 16 bytes on")
        if (lam.requires_grad or at is not None and weight.requires_grad) and torch.is_grad_enabled():
            raise ValueError("lam or weight asks for a gradient, and these calls have none: detach it, or call under "
                             "torch.no_grad()")
        d = self._diff
        d.lambda_, d.lambda_token, d.lambda_head = lam.data_ptr(), token, head
        d.weight, d.eps, d.gain = at, eps, gain
        work = step.diff_work(self)
        code = self._lib.agft_diff_attend(self._cfg, self.ptr, self.nbytes, tables.ptr, tables.nbytes, step.ptr,
                                          step.nbytes, n, step.max_new, self._b0, self._bdiff, self._b1,
                                          None if lse is None else lse.data_ptr(),
                                          1.0 / math.sqrt(c.dim) if scale is None else float(scale), work.data_ptr(),
                                          work.numel(), self._s())
        if code != L.AGFT_OK:
            L.check("agft_diff_attend", code)
        return out

    def copy(self, edit):
        """Copy the pages that a planned edit moves or fills, before or after its commit,
        but before the tables change again, behind the windows planned before it and
        ahead of this layer's tokens of later ones."""
        self._fits(edit, "edit")
        if edit._when != edit._of._changes or edit._number != edit._of._number and not edit._done:
            raise ValueError("the tables have changed since the edit was planned, or something else has been: its pages "
                             "may be others' by now")
        if self._appended > edit._number and self._appended_of is edit._of._token:
            raise ValueError("a later window's tokens are in this layer already: the edit's pages may be theirs")
        code = self._lib.agft_pages_copy(self._cfg, self.ptr, self.nbytes, edit.ptr, edit.nbytes, edit.max_moves, self._s())
        if code != L.AGFT_OK:
            L.check("agft_pages_copy", code)
        self._copied, self._copied_of = edit._number, edit._of._token

    def export(self, slots, dtype=torch.bfloat16):
        """Keys and values of the slots [n] (int64; -1 gives zeros) as two
        tensors [n][heads][dim] of dtype."""
        if slots.device != self.device or slots.dtype != torch.int64 or slots.dim() != 1 or not slots.is_contiguous():
            raise ValueError(f"slots must be a contiguous int64 tensor [n] on {self.device}")
        if dtype not in TYPES:
            raise ValueError(f"no exports in {dtype}")
        n, H, D = slots.numel(), self.cfg.heads, self.cfg.dim
        k, v = self._empty(2, n, H, D, dtype=dtype)
        if n:
            for d, t in ((self._d0, k), (self._d1, v)):
                d.data, d.token_stride, d.head_stride, d.type = t.data_ptr(), H * D, D, TYPES[dtype]
            code = self._lib.agft_kv_export(self._cfg, self.ptr, self.nbytes, slots.data_ptr(), n, self._b0, self._b1,
                                            self._s())
            if code != L.AGFT_OK:
                L.check("agft_kv_export", code)
        return k, v


HALVES = {t: c for t, c in TYPES.items() if t != torch.float32}
