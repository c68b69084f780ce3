"""Thin PyTorch binding of the paged key/value cache, of 16 or 8 bits, and its
attention (ewsjf_cache_*, ewsjf_prefix_plan, ewsjf_window_plan,
ewsjf_attention in include/ewsjf.h): what a server runs for the requests a
scheduling step admits, on the same card and stream.

    cache = kv.PagedCache.new(layers, n_pages, page_size, kv_heads, head_dim, n_slots, width)
    granted = cache.fork(parent, child, tokens)     # a prompt's pages shared, its partial page copied
    slot = torch.where(granted > 0, child, -1)      # a refused request has no slot in what follows
    granted = cache.extend(slot, new)               # pages for new tokens
    slot = torch.where(granted > 0, slot, -1)
    plan = kv.prefix_plan(cache, slot, q_start, group_start, shared, total_q=.., max_q=.., q_heads=..)
    cache.append(layer, k, v, slot, q_start, granted=granted)  # every layer: the new tokens' keys and values,
    out, lse = kv.attention(q, cache, layer, plan)             # and their queries, with the same plan
    granted = cache.reorder(slot, parent)           # beams: each slot takes over its parent's tokens
    k, v = cache.read(layer, slot, start, total=..) # what the pages stand for, dense
    cache.release(child)

Nothing here synchronizes the host; a request that does not fit the pool is
told by granted == 0 on the device.  A slot of -1 is refused, written nowhere
and released as nothing; its queries get out 0 and lse -inf.

Calls run on the current stream or on the one that is given.  With either on
another device than the cache's a call raises ValueError: nothing is launched.
"""
from __future__ import annotations

import contextlib
import ctypes as C

import torch

from . import _lib as L
from .ewsjf import Workspace, _need, _stream

_HERE = contextlib.nullcontext()
_DTYPES = {torch.bfloat16: L.BF16, torch.float16: L.F16}
_CODES = {torch.bfloat16: L.E4M3_BF16, torch.float16: L.E4M3_F16}


def _addr(struct) -> int:
    return C.addressof(struct)


def _stride(t: torch.Tensor, dim: int) -> int:
    """Stride in elements, 0 for a dim of size 1 (torch leaves any value there)."""
    return t.stride(dim) if t.shape[dim] > 1 else 0


def _new(stream, *args, dtype: torch.dtype, device) -> torch.Tensor:
    """A tensor that a call on `stream` writes: from that stream's memory (the current stream's may still be in use
    there), and kept from reuse until the current stream, where the caller has it, is done with it."""
    if stream is None:
        return torch.empty(*args, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        t = torch.empty(*args, dtype=dtype, device=device)
    t.record_stream(torch.cuda.current_stream(t.device))
    return t


def _keep(owner, raw: int, stream, *tensors: torch.Tensor) -> None:
    """The owner's tensors, which a call on the stream (raw: its handle) uses, are kept from reuse until the stream is
    done with them, whenever the owner lets go of them.  Only needed where the stream is not the last call's."""
    for t in tensors:
        t.record_stream(torch.cuda.current_stream(t.device) if stream is None else stream)
    owner.used_on = raw


def _scratch(ws: Workspace | None, nbytes: int, device, raw: int, stream) -> torch.Tensor:
    with _HERE if stream is None else torch.cuda.stream(stream):
        if ws is None:
            return torch.empty(max(256, nbytes), dtype=torch.uint8, device=device)
        before, buf = ws.buf, ws.get(nbytes)
    if raw != ws.used_on or buf is not before:
        _keep(ws, raw, stream, buf)
    return buf


def page_bytes(page_size: int, kv_heads: int, head_dim: int) -> int:
    """Bytes of a page's keys, or of its values, in an 8-bit cache (ewsjf_cache_page_bytes)."""
    n = int(L.lib().ewsjf_cache_page_bytes(page_size, kv_heads, head_dim, L.E4M3_BF16))
    if n == 0:
        raise ValueError("pages of these sizes are not supported (see ewsjf_cache)")
    return n


class PagedCache:
    """Pages of keys and values, the rows that name them and their counts.

    data: bfloat16 or float16 [layers][2][n_pages][kv_heads][page_size][head_dim],
    2 for keys and values; a page's block may also lie in memory as
    [page_size][kv_heads][head_dim] (give that tensor transposed).  refs: int32
    [n_pages], rows that hold a page, 0 for a free one.  table: int32
    [n_slots][width], a slot's pages, -1 for none.  length: int32 [n_slots],
    tokens held.

    In 8 bits (`of_bytes`, `new(bits=8)`) data is uint8
    [layers][2][n_pages][page_bytes], a page's e4m3 codes and behind them the
    exponents of their scales (`codes`, `scales`), and dtype is the 16-bit type
    of what is appended, read and attended with."""

    def __init__(self, data: torch.Tensor, refs: torch.Tensor, table: torch.Tensor, length: torch.Tensor):
        if not isinstance(data, torch.Tensor) or data.dtype not in _DTYPES or not data.is_cuda or data.dim() != 6 \
                or data.shape[1] != 2 or (data.shape[5] > 1 and data.stride(5) != 1):
            raise TypeError("data must be a CUDA tensor [layers][2][n_pages][kv_heads][page_size][head_dim] of bfloat16 "
                            "or float16")
        _need(refs, torch.int32, "refs")
        _need(table, torch.int32, "table")
        _need(length, torch.int32, "length")
        layers, _, n_pages, kv_heads, page_size, head_dim = data.shape
        self._hold(data, refs, table, length, [_stride(data, d) for d in range(5)],
                   (layers, n_pages, page_size, kv_heads, head_dim), data.dtype, _DTYPES[data.dtype])

    def _hold(self, data, refs, table, length, strides, sizes, dtype, code) -> None:
        layers, n_pages, page_size, kv_heads, head_dim = sizes
        if table.dim() != 2 or refs.shape != (n_pages,) or length.shape != (table.shape[0],):
            raise ValueError("refs has one entry per page, table and length one row per slot")
        if any(t.device != data.device for t in (refs, table, length)):
            raise ValueError("data, refs, table and length are on one device")
        self.data, self.refs, self.table, self.length = data, refs, table, length
        self.page_size, self.device, self.dtype = page_size, data.device, dtype
        self.used_on = None
        # what a plan's layout and slots follow
        self.sizes = (data.device, kv_heads, head_dim, page_size, *table.shape, code >= L.E4M3_BF16)
        self.c = L.Cache(data.data_ptr(), refs.data_ptr(), table.data_ptr(), length.data_ptr(), *strides,
                         layers, n_pages, page_size, kv_heads, head_dim, code, *table.shape)
        self._c = _addr(self.c)
        self._ws_bytes = int(L.lib().ewsjf_cache_workspace_bytes(self._c))
        self._reorder_bytes = {}  # by the number of slots
        if self._ws_bytes == 0:
            raise ValueError("a cache of these sizes or strides is not supported (see ewsjf_cache)")

    @classmethod
    def of(cls, data, refs, table, length) -> "PagedCache":
        """A cache over tensors that the caller holds."""
        return cls(data, refs, table, length)

    @classmethod
    def of_bytes(cls, data: torch.Tensor, refs: torch.Tensor, table: torch.Tensor, length: torch.Tensor,
                 page_size: int, kv_heads: int, head_dim: int, dtype: torch.dtype = torch.bfloat16,
                 tokens_first: bool = False) -> "PagedCache":
        """An 8-bit cache over tensors that the caller holds: data uint8
        [layers][2][n_pages][page_bytes(page_size, kv_heads, head_dim)], the
        last dim contiguous.  tokens_first: a page's codes lie as
        [page_size][kv_heads][head_dim]."""
        if dtype not in _CODES:
            raise TypeError("dtype is bfloat16 or float16: what the codes stand for")
        if not isinstance(data, torch.Tensor) or data.dtype != torch.uint8 or not data.is_cuda or data.dim() != 4 \
                or data.shape[1] != 2 or data.shape[3] != page_bytes(page_size, kv_heads, head_dim) \
                or data.stride(3) != 1:
            raise TypeError("data must be a CUDA tensor [layers][2][n_pages][page_bytes] of uint8")
        _need(refs, torch.int32, "refs")
        _need(table, torch.int32, "table")
        _need(length, torch.int32, "length")
        self = cls.__new__(cls)
        inner = (head_dim, kv_heads * head_dim) if tokens_first else (page_size * head_dim, head_dim)
        self._hold(data, refs, table, length, [_stride(data, d) for d in range(3)] + list(inner),
                   (data.shape[0], data.shape[2], page_size, kv_heads, head_dim), dtype, _CODES[dtype])
        return self

    @classmethod
    def new(cls, layers: int, n_pages: int, page_size: int, kv_heads: int, head_dim: int, n_slots: int, width: int,
            dtype: torch.dtype = torch.bfloat16, device=None, bits: int = 16) -> "PagedCache":
        """An empty cache: every page free, every slot without tokens.  bits: 16, or 8 for e4m3 codes."""
        if bits not in (8, 16):
            raise ValueError("bits is 16 or 8")
        dev = torch.device(device or "cuda")
        books = (torch.zeros(n_pages, dtype=torch.int32, device=dev),
                 torch.full((n_slots, width), -1, dtype=torch.int32, device=dev),
                 torch.zeros(n_slots, dtype=torch.int32, device=dev))
        if bits == 16:
            return cls(torch.zeros((layers, 2, n_pages, kv_heads, page_size, head_dim), dtype=dtype, device=dev), *books)
        data = torch.zeros((layers, 2, n_pages, page_bytes(page_size, kv_heads, head_dim)), dtype=torch.uint8, device=dev)
        return cls.of_bytes(data, *books, page_size, kv_heads, head_dim, dtype)

    @property
    def bits(self) -> int:
        return 8 if self.c.dtype >= L.E4M3_BF16 else 16

    @property
    def codes(self) -> torch.Tensor:
        """An 8-bit cache's codes, float8_e4m3fn [layers][2][n_pages][kv_heads][page_size][head_dim], in place."""
        c, n = self.c, self.c.kv_heads * self.c.page_size * self.c.head_dim
        if self.bits != 8:
            raise ValueError("a 16-bit cache has no codes")
        flat = self.data[..., :n].view(torch.float8_e4m3fn)
        if c.token_stride == c.head_dim or c.page_size == 1:
            return flat.unflatten(-1, (c.kv_heads, c.page_size, c.head_dim))
        return flat.unflatten(-1, (c.page_size, c.kv_heads, c.head_dim)).transpose(3, 4)

    @property
    def scales(self) -> torch.Tensor:
        """An 8-bit cache's scales, uint8 [layers][2][n_pages][kv_heads][page_size], in place: b stands for 2^(b - 127)."""
        c, n = self.c, self.c.kv_heads * self.c.page_size
        if self.bits != 8:
            raise ValueError("a 16-bit cache has no scales")
        return self.data[..., n * c.head_dim:n * (c.head_dim + 1)].unflatten(-1, (c.kv_heads, c.page_size))

    def _on(self, stream) -> int:
        """The handle of the stream that a call uses the cache on."""
        raw = _stream(stream)
        if stream is not None and stream.device != self.device or \
                stream is None and self.device.index not in (None, torch._C._cuda_getDevice()):
            raise ValueError("the cache is on another device than the call's stream")
        if raw != self.used_on:
            _keep(self, raw, stream, self.data, self.refs, self.table, self.length)
        return raw

    def _ids(self, t: torch.Tensor, name: str, n: int | None = None) -> int:
        if _need(t, torch.int32, name).device != self.device:
            raise ValueError(f"{name} is on another device than the cache")
        if n is not None and t.numel() != n:
            raise ValueError(f"{name} needs {n} entries")
        return t.data_ptr()

    def extend(self, slot: torch.Tensor, tokens: torch.Tensor, granted: torch.Tensor | None = None,
               ws: Workspace | None = None, stream=None) -> torch.Tensor:
        """Room for tokens[i] more tokens in slot[i]: int32 [n], 1 granted, 0
        refused (ewsjf_cache_extend)."""
        n = slot.numel()
        granted = _new(stream, n, dtype=torch.int32, device=self.device) if granted is None else granted
        raw = self._on(stream)
        buf = _scratch(ws, self._ws_bytes, self.device, raw, stream)
        L.check(L.lib().ewsjf_cache_extend(self._c, self._ids(slot, "slot"), self._ids(tokens, "tokens", n), n,
                                           self._ids(granted, "granted", n), buf.data_ptr(), buf.numel(),
                                           raw), "ewsjf_cache_extend")
        return granted

    def fork(self, parent: torch.Tensor, child: torch.Tensor, tokens: torch.Tensor,
             granted: torch.Tensor | None = None, ws: Workspace | None = None, stream=None) -> torch.Tensor:
        """child[i] := the first tokens[i] tokens of parent[i]: int32 [n], 1
        granted, 0 refused (ewsjf_cache_fork)."""
        n = child.numel()
        granted = _new(stream, n, dtype=torch.int32, device=self.device) if granted is None else granted
        raw = self._on(stream)
        buf = _scratch(ws, self._ws_bytes, self.device, raw, stream)
        L.check(L.lib().ewsjf_cache_fork(self._c, self._ids(parent, "parent", n), self._ids(child, "child"),
                                         self._ids(tokens, "tokens", n), n, self._ids(granted, "granted", n),
                                         buf.data_ptr(), buf.numel(), raw), "ewsjf_cache_fork")
        return granted

    def release(self, slot: torch.Tensor, begin: torch.Tensor | None = None, end: torch.Tensor | None = None,
                ws: Workspace | None = None, stream=None) -> None:
        """Empty the slots, or give up their pages that lie wholly in tokens
        [begin, end) (ewsjf_cache_release; ws is not used)."""
        n = slot.numel()
        b = None if begin is None else self._ids(begin, "begin", n)
        e = None if end is None else self._ids(end, "end", n)
        L.check(L.lib().ewsjf_cache_release(self._c, self._ids(slot, "slot"), b, e, n, self._on(stream)),
                "ewsjf_cache_release")

    def copy(self, src: torch.Tensor, dst: torch.Tensor, stream=None) -> None:
        """Pages src[j] to pages dst[j] in every layer (ewsjf_cache_copy)."""
        n = src.numel()
        L.check(L.lib().ewsjf_cache_copy(self._c, self._ids(src, "src"), self._ids(dst, "dst", n), n,
                                         self._on(stream)), "ewsjf_cache_copy")

    def compact(self, out=None, ws: Workspace | None = None, stream=None):
        """Move the used pages to the front: (table, refs, used[1]) of the
        compacted pool (ewsjf_cache_compact).  out: arrays for them, the
        cache's own table and refs for a compaction in place; otherwise the
        cache's arrays stay as they are and `adopt` takes the new ones."""
        if out is None:
            out = tuple(_new(stream, s, dtype=torch.int32, device=self.device)
                        for s in (self.table.shape, self.refs.shape, 1))
        table, refs, used = out
        raw = self._on(stream)
        buf = _scratch(ws, self._ws_bytes, self.device, raw, stream)
        L.check(L.lib().ewsjf_cache_compact(self._c, self._ids(table, "table", self.table.numel()),
                                            self._ids(refs, "refs", self.refs.numel()), self._ids(used, "used", 1),
                                            buf.data_ptr(), buf.numel(), raw), "ewsjf_cache_compact")
        return out

    def adopt(self, table: torch.Tensor, refs: torch.Tensor) -> None:
        """Take compact()'s table and refs as the cache's own."""
        self.c.table = self._ids(table, "table", self.table.numel())
        self.c.refs = self._ids(refs, "refs", self.refs.numel())
        self.table, self.refs, self.used_on = table.view_as(self.table), refs, None

    def append(self, layer: int, k: torch.Tensor, v: torch.Tensor, slot: torch.Tensor, q_start: torch.Tensor,
               stream=None, *, granted: torch.Tensor | None = None) -> None:
        """Write keys and values [total][kv_heads][head_dim] of the slots'
        newest tokens.  granted: what extend gave for these requests; nothing
        is written for a refused one (ewsjf_cache_append_granted).  None: for
        requests that were all granted; whole pages that other rows hold too
        are not written (ewsjf_cache_append)."""
        n, want = slot.numel(), (self.c.kv_heads, self.c.head_dim)
        for t, name in ((k, "k"), (v, "v")):
            if not isinstance(t, torch.Tensor) or t.dtype != self.dtype or t.device != self.device \
                    or t.dim() != 3 or tuple(t.shape[1:]) != want or t.stride(2) != 1 or t.shape != k.shape:
                raise TypeError(f"{name} must be a CUDA tensor [total][kv_heads][head_dim] of the cache's type")
        g = None if granted is None else self._ids(granted, "granted", n)
        L.check(L.lib().ewsjf_cache_append_granted(self._c, int(layer), k.data_ptr(), v.data_ptr(), _stride(k, 0),
                                                   _stride(k, 1), _stride(v, 0), _stride(v, 1),
                                                   self._ids(slot, "slot"), self._ids(q_start, "q_start", n + 1), g,
                                                   n, k.shape[0], self._on(stream)), "ewsjf_cache_append")


    def read(self, layer: int, slot: torch.Tensor, start: torch.Tensor, begin: torch.Tensor | None = None, *,
             total: int | None = None, out=None, stream=None):
        """Keys and values (k, v) [total][kv_heads][head_dim] of the slots'
        tokens, in 16 bits: rows [start[s], start[s + 1]) get the tokens of
        slot[s] from begin[s] on (None: 0), zeros where there is none
        (ewsjf_cache_read).  out: (k, v) to write into, whose rows past the
        last sequence's stay as they are; otherwise `total` rows are made,
        those past the last sequence's zeros (ewsjf_cache_read_all)."""
        n, want, read = slot.numel(), (self.c.kv_heads, self.c.head_dim), L.lib().ewsjf_cache_read
        if out is None:
            read = L.lib().ewsjf_cache_read_all
            if total is None:
                raise ValueError("total or out is needed")
            k, v = out = tuple(_new(stream, (int(total), *want), dtype=self.dtype, device=self.device) for _ in range(2))
        else:
            k, v = out
            for t, name in ((k, "k"), (v, "v")):
                if _need(t, self.dtype, name).dim() != 3 or tuple(t.shape[1:]) != want or t.shape != k.shape \
                        or t.device != self.device:
                    raise ValueError(f"{name} is [total][kv_heads][head_dim] on the cache's device")
            if total is not None and total != k.shape[0]:
                raise ValueError("out has total rows")
        b = None if begin is None else self._ids(begin, "begin", n)
        L.check(read(self._c, int(layer), self._ids(slot, "slot"), self._ids(start, "start", n + 1), b, n, k.shape[0],
                     k.data_ptr(), v.data_ptr(), self._on(stream)), "ewsjf_cache_read")
        return out

    def reorder(self, slot: torch.Tensor, parent: torch.Tensor, granted: torch.Tensor | None = None,
                ws: Workspace | None = None, stream=None) -> torch.Tensor:
        """slot[i] := what slot[parent[i]] held, for all i at once; a parent of
        -1 empties the slot.  int32 [n], 1 for a slot that holds its parent's
        tokens, else 0 (ewsjf_cache_reorder)."""
        n = slot.numel()
        granted = _new(stream, n, dtype=torch.int32, device=self.device) if granted is None else granted
        nbytes = self._reorder_bytes.get(n)
        if nbytes is None:
            nbytes = self._reorder_bytes[n] = int(L.lib().ewsjf_cache_reorder_workspace_bytes(self._c, n))
        raw = self._on(stream)
        buf = _scratch(ws, nbytes, self.device, raw, stream)
        L.check(L.lib().ewsjf_cache_reorder(self._c, self._ids(slot, "slot"), self._ids(parent, "parent", n), n,
                                            self._ids(granted, "granted", n), buf.data_ptr(), buf.numel(), raw),
                "ewsjf_cache_reorder")
        return granted


class AttentionPlan:
    """What follows from a batch's lengths, on the device; serves every layer
    of a step (prefix_plan, window_plan), of its cache or of one with the same
    sizes, slots and lengths."""

    def __init__(self, cache: PagedCache, batch: L.Batch, stream=None):
        self.b = batch
        self.sizes = cache.sizes
        self.q_shape = (batch.total_q, batch.q_heads, cache.c.head_dim)
        self._b = _addr(batch)
        lib = L.lib()
        nbytes = int(lib.ewsjf_attention_plan_bytes(cache._c, self._b))
        if nbytes == 0:
            raise ValueError("a batch of these sizes is not supported (see ewsjf_batch)")
        self.ws_bytes = int(lib.ewsjf_attention_workspace_bytes(cache._c, self._b))
        self.buf = _new(stream, nbytes, dtype=torch.uint8, device=cache.device)
        self.used_on = _stream(stream)


def prefix_plan(cache: PagedCache, slot: torch.Tensor, q_start: torch.Tensor, group_start: torch.Tensor | None,
                shared: torch.Tensor | None, *, total_q: int, max_q: int, q_heads: int, stream=None) -> AttentionPlan:
    """Plan for sequences slot[s] with query tokens [q_start[s], q_start[s +
    1]) whose groups [group_start[g], group_start[g + 1]) share their first
    shared[g] tokens (ewsjf_prefix_plan); group_start = shared = None: nothing
    is shared."""
    n, groups = slot.numel(), 0 if shared is None else shared.numel()
    gs = None if shared is None else cache._ids(group_start, "group_start", groups + 1)
    sh = None if shared is None else cache._ids(shared, "shared")
    plan = AttentionPlan(cache, L.Batch(n, groups, int(total_q), int(max_q), int(q_heads), 0, 0), stream)
    L.check(L.lib().ewsjf_prefix_plan(cache._c, plan._b, cache._ids(slot, "slot"),
                                      cache._ids(q_start, "q_start", n + 1), gs, sh, plan.buf.data_ptr(),
                                      plan.buf.numel(), cache._on(stream)), "ewsjf_prefix_plan")
    return plan


def window_plan(cache: PagedCache, slot: torch.Tensor, q_start: torch.Tensor, window: int, sinks: int = 0, *,
                total_q: int, max_q: int, q_heads: int, stream=None) -> AttentionPlan:
    """Plan for sequences slot[s] with query tokens [q_start[s], q_start[s +
    1]) that see the last `window` tokens and the first `sinks`
    (ewsjf_window_plan)."""
    n = slot.numel()
    plan = AttentionPlan(cache, L.Batch(n, 0, int(total_q), int(max_q), int(q_heads), int(window), int(sinks)), stream)
    L.check(L.lib().ewsjf_window_plan(cache._c, plan._b, cache._ids(slot, "slot"),
                                      cache._ids(q_start, "q_start", n + 1), plan.buf.data_ptr(), plan.buf.numel(),
                                      cache._on(stream)), "ewsjf_window_plan")
    return plan


def attention(q: torch.Tensor, cache: PagedCache, layer: int, plan: AttentionPlan, scale: float | None = None,
              out: torch.Tensor | None = None, lse: torch.Tensor | None = None, ws: Workspace | None = None,
              stream=None):
    """Attention of q [total_q][q_heads][head_dim] (dims contiguous, other
    strides free) over one layer: (out, lse), lse float32
    [total_q][q_heads] the ln of the softmax's sum (ewsjf_attention).  scale
    defaults to head_dim ** -0.5."""
    shape = plan.q_shape
    if plan.sizes != cache.sizes:
        raise ValueError("the plan is of a cache with other sizes")
    if not isinstance(q, torch.Tensor) or q.dtype != cache.dtype or q.device != cache.device or q.shape != shape \
            or q.stride(2) != 1:
        raise TypeError(f"q must be a CUDA tensor {shape} of the cache's type with contiguous dims")
    if out is None:
        out = _new(stream, shape, dtype=q.dtype, device=q.device)
    elif _need(out, q.dtype, "out").shape != q.shape:
        raise ValueError("out has q's shape")
    if lse is None:
        lse = _new(stream, shape[:2], dtype=torch.float32, device=q.device)
    elif _need(lse, torch.float32, "lse").shape != q.shape[:2]:
        raise ValueError("lse is [total_q][q_heads]")
    raw = cache._on(stream)
    if raw != plan.used_on:
        _keep(plan, raw, stream, plan.buf)
    buf = _scratch(ws, plan.ws_bytes, cache.device, raw, stream)
    L.check(L.lib().ewsjf_attention(cache._c, plan._b, int(layer), q.data_ptr(), _stride(q, 0), _stride(q, 1),
                                    shape[2] ** -0.5 if scale is None else float(scale), plan.buf.data_ptr(),
                                    out.data_ptr(), lse.data_ptr(), buf.data_ptr(), buf.numel(), raw), "ewsjf_attention")
    return out, lse
