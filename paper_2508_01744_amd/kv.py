"""Python front end of the serving node's paged cache (agft_kv.h): torch
supplies device memory and streams, the work runs in the HIP kernels behind
libagft.so.

One window of a node with a KvTables `tables` and, per layer, a KvCache `cache`:

    step = tables.plan(add, max_tokens)        # pages and slots of the new tokens
    cache.append(step, k, v)                   # per layer
    out = cache.attend(tables, step, q)        # per layer
    tables.commit(step)                        # the new lengths become the tables'

Calls enqueue on the stream given to the object, or else on the stream that is
current when they are called; nothing here waits for the GPU except load().
There is no backward pass: tensors that ask for a gradient are refused.
Launches go to the calling thread's current device, which has to be the object's.
Tensors of another stream are the caller's to order, as for any torch call.
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
        if t.device != self.device or t.dtype != torch.int32 or not t.is_contiguous() or tuple(t.shape) != shape:
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
        self.planned = False

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


class KvTables(_OnStream):
    """Block tables, lengths and the ring of free pages of a node's requests:
    counters [8], lengths [R], table [R][row_pages], ring [pages] (int32)."""
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
        self.reset()

    def reset(self):
        """No request holds a token, every page is free."""
        L.check("agft_kv_reset", self._lib.agft_kv_reset(self._cfg, self.ptr, self.nbytes, self._s()))

    def load(self, lengths, table, free):
        """Take over the tables of a running node: lengths [R], table
        [R][row_pages] and the free pages in the order of their use (int32).
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
        counters = torch.tensor([0, free.numel(), 0, 0, 0, 0, 0, 0], dtype=torch.int32)
        with self._settled():
            self.lengths.copy_(lengths)
            self.table.copy_(table)
            self.ring.zero_()
            self.ring[:free.numel()].copy_(free)
            self.counters.copy_(counters)

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
        code = self._lib.agft_kv_plan(self._cfg, self.ptr, self.nbytes, add.data_ptr(), step.ptr, step.nbytes,
                                      step.max_tokens, self._s())
        if code != L.AGFT_OK:
            L.check("agft_kv_plan", code)
        step.planned = True
        return step

    def commit(self, step):
        """The planned window's lengths and free pages become the tables'."""
        self._fits(step, "step")
        L.check("agft_kv_commit", self._lib.agft_kv_commit(self._cfg, self.ptr, self.nbytes, step.ptr, step.nbytes,
                                                           step.max_tokens, self._s()))


class KvCache(_OnStream):
    """One layer's pages: 8-bit codes and an exponent per page, head and side."""

    def __init__(self, cfg, device="cuda", stream=None):
        self._init(cfg, device, stream)
        # what calls tell the library of their tensors (a front end is not thread-safe, like a Tuner)
        self._d0, self._d1 = L.agft_kv_dense(), L.agft_kv_dense()
        self._b0, self._b1 = ctypes.byref(self._d0), ctypes.byref(self._d1)
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

    def _dense(self, d, t, heads, rows, what, types=TYPES):
        """Fill the agft_kv_dense d from a [tokens][heads][dim] tensor of at least `rows` tokens."""
        try:
            n, h, dim = t.shape
            token, head, one = t.stride()
            kind = types[t.dtype]
        except (ValueError, KeyError):
            n = h = dim = one = -1
        if n < rows or h != heads or dim != self.cfg.dim or one != 1 or t.get_device() != self._index:
            raise ValueError(f"{what} must be [{rows} or more][{heads}][{self.cfg.dim}] on {self.device}, "
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
        self._fits(step, "step")
        if k.dtype != v.dtype:
            raise ValueError("k and v must have one type")
        self._dense(self._d0, k, H, n, "k")
        self._dense(self._d1, v, H, n, "v")
        code = self._lib.agft_kv_append(self._cfg, self.ptr, self.nbytes, step.ptr, step.nbytes, n, self._b0, self._b1,
                                        self._s())
        if code != L.AGFT_OK:
            L.check("agft_kv_append", code)

    def attend(self, tables, step, q, out=None, lse=None, scale=None):
        """softmax(scale q K^T) V of the window's tokens over their requests'
        tokens up to themselves.  q, out [max_tokens][heads * group][dim], bf16
        or fp16 (out is allocated if None; rows past the window's tokens stay as
        they are, in a fresh one whatever its memory held); lse float32
        [max_tokens][heads * group] or None receives the logarithms of the sums;
        scale: 1 / sqrt(dim) if None."""
        c, n = self.cfg, step.max_tokens
        hq = c.heads * c.group
        self._fits(step, "step")
        self._fits(tables, "tables")
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
