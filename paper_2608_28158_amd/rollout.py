"""Generation over a rollout forest: a paged key/value cache, attention of new
rows over its segments, and the recurrent steps of the linear layers.  Argument
marshalling around harts_cache_*, harts_gen_* and harts_*_step of libharts.so;
every step runs in the library's kernels, on the current stream of the
tensors' device.  The calls check their arguments and launch in a compiled
binding (csrc/rollout_ext.cpp): a token is many small ones.

A forest here is what the batch in flight looks like: a segment is a run of
rows that its descendants share (a prompt, a branch, the tail of one rollout),
and sequences are the chains from a root to a leaf.  Segment ids are the
cache's; a fork of a sequence is two new segments below it, with no row copied.

    cache = RolloutCache(n_pages, n_seg, pitch, heads, d, kind="e4m3", layers=24)
    cache.reserve(seg, rows)                       # pages, ahead of the rows
    batch = RolloutBatch(cache, parent, n_new, q_heads)
    batch.advance()                                # once per step: lengths grow by n_new
    batch.write(k, v, layer)                       # per layer: the new rows enter the cache
    o, lse = batch.attend(q, layer)                # and their queries see it

A batch's tables serve every step until the forest or n_new changes, so a step
can be captured into a graph and replayed while the lengths grow, for as long
as the program keeps the batch and the cache.  Nothing here
is differentiable: inputs that require a gradient are refused while gradients
are recorded, and inputs that carry a tangent (the training forms are tree_la,
KdaRunner and harts_attn_*).  What a call writes counts as modified.
"""
from __future__ import annotations

import ctypes as C

import numpy as np
import torch

from . import _lib

PAGE = 64


def _device(device):
    d = torch.device(device)
    if d.type != "cuda":
        raise RuntimeError("generation runs on the GPU only")
    return d if d.index is not None else torch.device("cuda", torch.cuda.current_device())


# The current stream's handle without a Stream object around it (0.1 us instead
# of 1.2, of a small call's 5), where torch offers that.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
    (lambda index: torch.cuda.current_stream(index).cuda_stream)


def _host_table(name, values, n, dtype):
    """A table of one number for each of n segments, in a type that holds them as they are."""
    given = np.asarray(values)
    if given.shape != (n,):
        raise ValueError(f"{name} must have one entry for each of the cache's {n} segments")
    with np.errstate(invalid="ignore"):
        a = np.ascontiguousarray(given, dtype=dtype)
    if not np.array_equal(a, given):
        raise ValueError(f"{name} must hold whole numbers of {np.dtype(dtype).name}")
    return a


class _OnStreams:
    """An object with tensors that calls on any stream may use: their memory is
    not handed out again before what those streams had queued when the object
    was dropped has run.  ``_known`` are the streams it has been used on."""

    def _keep(self, index, tensors):
        self._index, self._kept = index, tensors
        self._known = {_raw_stream(index)}           # (theirs, by the allocator)

    def _meet(self, stream):
        for t in self._kept:
            t.record_stream(torch.cuda.current_stream(self._index))
        self._known.add(stream)

    def _stream(self):
        """The current stream, known from now on."""
        stream = _raw_stream(self._index)
        if stream not in self._known:
            self._meet(stream)
        return stream


class RolloutCache(_OnStreams):
    """Paged keys and values of ``layers`` layers (harts_cache): ``n_pages``
    pages of 64 rows shared by ``n_seg`` segments of up to ``pitch`` pages.
    kind "bf16" or "e4m3".  The tensors are the cache: k, v
    [layers, n_pages, heads, 64, d], k_exp, v_exp [layers, n_pages, heads, 64]
    (e4m3), pages [n_seg, pitch] and len [n_seg] int32."""

    def __init__(self, n_pages: int, n_seg: int, pitch: int, heads: int, d: int, kind: str = "bf16",
                 layers: int = 1, device="cuda"):
        if kind not in ("bf16", "e4m3"):
            raise ValueError("kind must be 'bf16' or 'e4m3'")
        if min(n_pages, n_seg, pitch, heads, layers) < 1 or d not in (64, 128):
            raise ValueError("need at least one page, segment, column, head and layer, and d in {64, 128}")
        if max(n_pages, n_seg, pitch) > 2 ** 31 - 1 or heads > 65535:
            raise ValueError("need at most 2^31 - 1 pages, segments and columns, and 65535 heads")
        self.L, self._ext, self.device = _lib.rollout(), _lib.rollout_binding(), _device(device)
        self.n_pages, self.n_seg, self.pitch, self.heads, self.d = n_pages, n_seg, pitch, heads, d
        self.kind, self.layers = kind, layers
        dt = torch.bfloat16 if kind == "bf16" else torch.float8_e4m3fn
        shape = (layers, n_pages, heads, PAGE, d)
        self.k = torch.empty(shape, dtype=dt, device=self.device)
        self.v = torch.empty(shape, dtype=dt, device=self.device)
        self.k_exp = self.v_exp = None
        if kind == "e4m3":
            self.k_exp = torch.empty(shape[:-1], dtype=torch.uint8, device=self.device)
            self.v_exp = torch.empty(shape[:-1], dtype=torch.uint8, device=self.device)
        self.pages = torch.full((n_seg, pitch), -1, dtype=torch.int32, device=self.device)
        self.len = torch.zeros(n_seg, dtype=torch.int32, device=self.device)
        self._free = list(range(n_pages - 1, -1, -1))
        self._held = [[] for _ in range(n_seg)]
        code = _lib.HARTS_BF16 if kind == "bf16" else _lib.HARTS_E4M3
        ptr = lambda t, i: None if t is None else t[i].data_ptr()
        fixed = (self.pages.data_ptr(), self.len.data_ptr(), n_pages, n_seg, pitch, heads, d, code)
        # (the library's view of each layer: the tensors above are written, never replaced)
        self._layers = [_lib.Cache(*(ptr(t, i) for t in (self.k, self.v, self.k_exp, self.v_exp)), *fixed)
                        for i in range(layers)]
        self._desc = [C.addressof(c) for c in self._layers]
        self._cells = tuple(t for t in (self.k, self.v, self.k_exp, self.v_exp) if t is not None)
        self._keep(self.device.index, self._cells + (self.pages, self.len))

    # -- pages (host bookkeeping) --------------------------------------------
    @property
    def free_pages(self):
        return len(self._free)

    def _seg(self, seg):
        if not 0 <= seg < self.n_seg:
            raise ValueError(f"segment {seg} outside [0, {self.n_seg})")
        return seg

    def reserve(self, seg: int, rows: int):
        """Pages for the segment's first ``rows`` rows (those it has are kept)."""
        held = self._held[self._seg(seg)]
        need = -(-rows // PAGE)
        if need > self.pitch:
            raise ValueError(f"{rows} rows need {need} pages, a segment has at most {self.pitch}")
        more = need - len(held)
        if more <= 0:
            return
        if more > len(self._free):
            raise RuntimeError(f"the cache is full: {more} pages wanted, {len(self._free)} free")
        self._stream()
        new = [self._free.pop() for _ in range(more)]
        self.pages[seg, len(held):need] = torch.tensor(new, dtype=torch.int32, device=self.device)
        held.extend(new)

    def release(self, seg: int):
        """Give the segment's pages back; it is empty afterwards."""
        held = self._held[self._seg(seg)]
        self._stream()
        self.pages[seg].fill_(-1)
        self.len[seg].zero_()
        self._free.extend(reversed(held))
        held.clear()

    def held_rows(self):
        """Rows [n_seg] that the reserved pages hold; of a cache without any, whose table the caller
        fills itself, the table's columns for every segment."""
        if not any(self._held):
            return np.full(self.n_seg, self.pitch * PAGE, np.int64)
        return np.array([len(held) * PAGE for held in self._held], np.int64)

    # -- rows ----------------------------------------------------------------
    def desc(self, layer: int):
        if not 0 <= layer < self.layers:
            raise ValueError(f"layer {layer} outside [0, {self.layers})")
        return self._desc[layer]

    def write(self, rows, k, v, layer: int = 0):
        """Rows k, v [n, heads, d] (bf16) into the cache at ``rows`` [n, 2]
        (int32 segment and position, negative from the segment's end).  A row
        may be named once; entries that name no existing row are skipped."""
        self._ext.cache_write(self.desc(layer), self._index, self._stream(), self._cells, rows, k, v)

    def read(self, rows, layer: int = 0):
        """(k, v) [n, heads, d] bf16: what the rows stand for, zeros where an
        entry names no existing row."""
        return self._ext.cache_read(self.desc(layer), self._index, self._stream(), rows)


class RolloutBatch(_OnStreams):
    """The new rows of one step over a cache's forest (harts_gen_tables).

    parent [n_seg]: parent segment or -1; n_new [n_seg]: query rows at the end
    of every segment (0 for those that only serve others, or are unused).
    capacity [n_seg]: about how many rows the segments hold while the batch is
    in use.  Results differ by rounding only, times by much more: the chip is
    shared out by capacities, so that room which stays empty is taken from the
    segments that all wait for.  (One token of 64 samples of a 65,000-row
    8-bit prefix, tails up to 3,900: 140 us by the present lengths, 556 with
    room for 32,768 more rows a tail, 728 with room for 65,000.)  Default:
    what the pages reserved by now hold; where much more is reserved than
    filled, pass the present lengths and make the batch anew now and then.
    Query rows are ordered by segment id, each segment's in order: ``rows`` is
    their table."""

    def __init__(self, cache: RolloutCache, parent, n_new, q_heads: int, capacity=None):
        self.cache, self.q_heads, self.L = cache, int(q_heads), cache.L
        if self.q_heads != q_heads or self.q_heads > 65535:
            raise ValueError(f"q_heads must be a whole number of at most 65535, got {q_heads}")
        parent = _host_table("parent", parent, cache.n_seg, np.int32)
        new = _host_table("n_new", n_new, cache.n_seg, np.int32)
        cap = cache.held_rows() if capacity is None else _host_table("capacity", capacity, cache.n_seg, np.int64)
        host = (cache.n_seg, parent.ctypes.data, new.ctypes.data, cap.ctypes.data, self.q_heads, cache.heads)
        self.sizes = _lib.GenSizes()
        _lib.check(self.L.harts_gen_layout(*host, C.byref(self.sizes)), "harts_gen_layout")
        self.n_rows = int(self.sizes.n_rows)
        # one upload: rows, order, items, part offsets and new rows, each from a multiple of 16 bytes
        shapes = ((self.n_rows, 2), (self.n_rows,), (self.sizes.n_items, 12), (self.n_rows + 1,), (cache.n_seg,))
        at = np.cumsum([0] + [-(-int(np.prod(s)) // 4) * 4 for s in shapes])
        host_tab = np.zeros(int(at[-1]), np.int32)
        part = lambda t: [t[i:i + int(np.prod(s))].reshape(s) for i, s in zip(at, shapes)]
        rows, order, items, off, n_new = part(host_tab)
        n_new[:] = new
        _lib.check(self.L.harts_gen_tables(*host, rows.ctypes.data, order.ctypes.data, items.ctypes.data,
                                           off.ctypes.data), "harts_gen_tables")
        self._tab = torch.from_numpy(host_tab).to(cache.device)
        cache._stream()
        self._keep(cache._index, (self._tab,))
        self.rows, order, items, off, self.n_new = part(self._tab)
        size = C.c_size_t()
        _lib.check(self.L.harts_gen_workspace_size(C.byref(self.sizes), self.q_heads, cache.d, C.byref(size)),
                   "harts_gen_workspace_size")
        self.ws_bytes = size.value
        self._call = (C.addressof(self.sizes), items.data_ptr(), order.data_ptr(), off.data_ptr(), self.q_heads,
                      self.ws_bytes, cache.device.index)

    def _meet(self, stream):
        super()._meet(stream)
        self.cache._stream()                         # (so the cache knows all streams that the batch does)

    def advance(self):
        """The segments' lengths grow by their new rows."""
        self._stream()
        self.cache.len.add_(self.n_new)

    def write(self, k, v, layer: int = 0):
        """The new rows' keys and values [n_rows, heads, d] into the cache."""
        c = self.cache
        c._ext.cache_write(c.desc(layer), c._index, self._stream(), c._cells, self.rows, k, v)

    def attend(self, q, layer: int = 0, scale=None, out=None):
        """(o [n_rows, q_heads, d] bf16, lse [n_rows, q_heads] float32) of the
        new rows' queries; scale defaults to d ** -0.5."""
        c = self.cache
        return c._ext.attend(c.desc(layer), *self._call, self._stream(), q, scale, out)


def la_step(q, k, v, g, S, S_out=None, idx_in=None, idx_out=None, row_off=None, scale=None, out=None):
    """Tokens of linear attention with scalar decay, one row of q, k, v
    [rows, H, d] and g [rows, H] for each sequence, or sequence i's rows
    [row_off[i], row_off[i + 1]) one after the other.  States start from
    S[idx_in[i]] and end in S_out[idx_out[i]] (no index: i; no S_out: in
    place).  Several sequences may start from one state: a fork.  A slot named
    again by idx_out gets no second state, and that sequence's outputs are NaN
    (the test is quadratic in sequences: free up to thousands, a quarter of the
    call at 16,384).  Returns o; rows that no sequence names keep what ``out``
    held, and without ``out`` they are uninitialised."""
    return _lib.rollout_binding().step(False, q, k, v, g, None, S, S_out, idx_in, idx_out, row_off, scale, out,
                                       _raw_stream)


def kda_step(q, k, v, g, beta, S, S_out=None, idx_in=None, idx_out=None, row_off=None, scale=None, out=None):
    """The same for KDA: g [rows, H, d], beta [rows, H]."""
    return _lib.rollout_binding().step(True, q, k, v, g, beta, S, S_out, idx_in, idx_out, row_off, scale, out,
                                       _raw_stream)
