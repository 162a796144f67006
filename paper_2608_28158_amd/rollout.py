"""Generation over a rollout forest: a paged key/value cache, attention of new
rows over its segments, and the recurrent steps of the linear layers.  Argument
marshalling around harts_cache_*, harts_gen_* and harts_*_step of libharts.so;
every step runs in the library's kernels, on the current stream of the
tensors' device.

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
can be captured into a graph and replayed while the lengths grow.  Nothing here
is differentiable: inputs that require a gradient are refused while gradients
are recorded (the training forms are tree_la, KdaRunner and harts_attn_*).
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


# The current stream's handle and device without the objects and the lazy
# initialisation around them (0.2 us instead of 1.4, of a small call's 7), where
# torch offers that.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
    (lambda index: torch.cuda.current_stream(index).cuda_stream)
_current = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _call(index, what, fn, *args):
    """fn(*args, stream) on the tensors' device: the library launches on the current one."""
    if _current() == index:
        code = fn(*args, _raw_stream(index))
    else:
        with torch.cuda.device(index):
            code = fn(*args, _raw_stream(index))
    if code:
        _lib.check(code, what)


def _check(shape, dtype, device, names, *tensors):
    """Contiguous tensors of one shape, type and device, none of them recording a gradient."""
    for t in tensors:
        if (t.dtype is not dtype or t.shape != shape or not t.is_contiguous() or t.device != device or
                t.requires_grad):
            break
    else:
        return
    for name, t in zip(names.split(), tensors):
        if t.dtype is not dtype or t.shape != shape or not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous {dtype} {list(shape)}, got {t.dtype} {list(t.shape)}"
                             f"{'' if t.is_contiguous() else ' with strides ' + str(t.stride())}")
        if t.device != device:
            raise ValueError(f"{name} is on {t.device}, expected {device}")
        if t.requires_grad and torch.is_grad_enabled():
            raise RuntimeError(f"{name} requires a gradient; generation is not differentiable")


class RolloutCache:
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
        self.L, self.device = _lib.rollout(), _device(device)
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
        self._desc = [C.byref(_lib.Cache(*(ptr(t, i) for t in (self.k, self.v, self.k_exp, self.v_exp)), *fixed))
                      for i in range(layers)]

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
        new = [self._free.pop() for _ in range(more)]
        self.pages[seg, len(held):need] = torch.tensor(new, dtype=torch.int32, device=self.device)
        held.extend(new)

    def release(self, seg: int):
        """Give the segment's pages back; it is empty afterwards."""
        held = self._held[self._seg(seg)]
        self.pages[seg].fill_(-1)
        self.len[seg].zero_()
        self._free.extend(reversed(held))
        held.clear()

    # -- rows ----------------------------------------------------------------
    def desc(self, layer: int):
        if not 0 <= layer < self.layers:
            raise ValueError(f"layer {layer} outside [0, {self.layers})")
        return self._desc[layer]

    def write(self, rows, k, v, layer: int = 0):
        """Rows k, v [n, heads, d] (bf16) into the cache at ``rows`` [n, 2]
        (int32 segment and position, negative from the segment's end).  A row
        may be named once; entries that name no existing row are skipped."""
        n = rows.shape[0]
        _check((n, 2), torch.int32, self.device, "rows", rows)
        _check((n, self.heads, self.d), torch.bfloat16, self.device, "k v", k, v)
        _call(self.device.index, "harts_cache_write", self.L.harts_cache_write, self.desc(layer), rows.data_ptr(), n,
              k.data_ptr(), v.data_ptr())

    def read(self, rows, layer: int = 0):
        """(k, v) [n, heads, d] bf16: what the rows stand for, zeros where an
        entry names no existing row."""
        n = rows.shape[0]
        _check((n, 2), torch.int32, self.device, "rows", rows)
        k = torch.empty((n, self.heads, self.d), dtype=torch.bfloat16, device=self.device)
        v = torch.empty_like(k)
        _call(self.device.index, "harts_cache_read", self.L.harts_cache_read, self.desc(layer), rows.data_ptr(), n,
              k.data_ptr(), v.data_ptr())
        return k, v


class RolloutBatch:
    """The new rows of one step over a cache's forest (harts_gen_tables).

    parent [n_seg]: parent segment or -1; n_new [n_seg]: query rows at the end
    of every segment (0 for those that only serve others, or are unused).
    capacity [n_seg]: rows that the segments may reach while the batch is in
    use, a hint for splitting long ones (default: the pitch).  Query rows are
    ordered by segment id, each segment's in order: ``rows`` is their table."""

    def __init__(self, cache: RolloutCache, parent, n_new, q_heads: int, capacity=None):
        self.cache, self.q_heads, self.L = cache, int(q_heads), cache.L
        parent = np.ascontiguousarray(parent, dtype=np.int32)
        new = np.ascontiguousarray(n_new, dtype=np.int32)
        cap = np.full(cache.n_seg, cache.pitch * PAGE, np.int64) if capacity is None else \
            np.ascontiguousarray(capacity, dtype=np.int64)
        for name, a in (("parent", parent), ("n_new", new), ("capacity", cap)):
            if a.shape != (cache.n_seg,):
                raise ValueError(f"{name} must have one entry for each of the cache's {cache.n_seg} segments")
        host = (cache.n_seg, parent.ctypes.data, new.ctypes.data, cap.ctypes.data, self.q_heads, cache.heads)
        self.sizes = _lib.GenSizes()
        _lib.check(self.L.harts_gen_layout(*host, C.byref(self.sizes)), "harts_gen_layout")
        self.n_rows = int(self.sizes.n_rows)
        rows, order = np.zeros((self.n_rows, 2), np.int32), np.zeros(self.n_rows, np.int32)
        items, off = np.zeros((self.sizes.n_items, 12), np.int32), np.zeros(self.n_rows + 1, np.int32)
        _lib.check(self.L.harts_gen_tables(*host, rows.ctypes.data, order.ctypes.data, items.ctypes.data,
                                           off.ctypes.data), "harts_gen_tables")
        dev = lambda a: torch.from_numpy(a).to(cache.device)
        self.rows, self._order, self._items, self._off, self.n_new = dev(rows), dev(order), dev(items), dev(off), dev(new)
        size = C.c_size_t()
        _lib.check(self.L.harts_gen_workspace_size(C.byref(self.sizes), self.q_heads, cache.d, C.byref(size)),
                   "harts_gen_workspace_size")
        self.ws_bytes = size.value
        # shapes to allocate by: one element each, expanded (0.5 us less a call than a shape and a type)
        like = lambda shape, dtype: torch.empty(1, dtype=dtype, device=cache.device).expand(shape)
        self._lse, self._ws = like((self.n_rows, self.q_heads), torch.float32), like((self.ws_bytes,), torch.uint8)
        self._shape = torch.Size((self.n_rows, self.q_heads, cache.d))
        self._tables = (C.byref(self.sizes), self._items.data_ptr(), self._order.data_ptr(), self._off.data_ptr(),
                        self.q_heads)

    def advance(self):
        """The segments' lengths grow by their new rows."""
        self.cache.len.add_(self.n_new)

    def write(self, k, v, layer: int = 0):
        """The new rows' keys and values [n_rows, heads, d] into the cache."""
        self.cache.write(self.rows, k, v, layer)

    def attend(self, q, layer: int = 0, scale=None, out=None):
        """(o [n_rows, q_heads, d] bf16, lse [n_rows, q_heads] float32) of the
        new rows' queries; scale defaults to d ** -0.5."""
        c = self.cache
        _check(self._shape, torch.bfloat16, c.device, "q", q)
        if out is None:
            out = torch.empty_like(q)
        else:
            _check(self._shape, torch.bfloat16, c.device, "out", out)
        # (from the allocator at every call: calls on other streams, or captured into other graphs, share none)
        lse = torch.empty_like(self._lse)
        ws = torch.empty_like(self._ws) if self.ws_bytes else None
        _call(c.device.index, "harts_gen_attn", self.L.harts_gen_attn, c.desc(layer), *self._tables,
              c.d ** -0.5 if scale is None else scale, q.data_ptr(), out.data_ptr(), lse.data_ptr(), _ptr(ws),
              self.ws_bytes)
        return out, lse


def _ptr(t):
    return None if t is None else t.data_ptr()


def _step(kda, q, k, v, g, beta, S, S_out, idx_in, idx_out, row_off, scale, out):
    shape, dtype, dev = q.shape, q.dtype, q.device
    if len(shape) != 3 or (dtype is not torch.bfloat16 and dtype is not torch.float32):
        raise ValueError("q must be float32 or bfloat16 [rows, H, d]")
    if dev.type != "cuda":
        raise RuntimeError("generation runs on the GPU only")
    n_rows, H, d = shape
    if out is None:
        _check(shape, dtype, dev, "q k v", q, k, v)
        out = torch.empty_like(q)
    else:
        _check(shape, dtype, dev, "q k v out", q, k, v, out)
    _check(shape if kda else (n_rows, H), torch.float32, dev, "g", g)
    if kda:
        _check((n_rows, H), torch.float32, dev, "beta", beta)
    n_seq = n_rows
    if row_off is not None:
        n_seq = row_off.numel() - 1
        if n_seq < 0:
            raise ValueError("row_off has one entry more than there are sequences")
        _check((n_seq + 1,), torch.int32, dev, "row_off", row_off)
    if S_out is None:
        if idx_out is not None:
            raise ValueError("an update in place leaves every state where it was: idx_out has to be None")
        S_out, idx_out = S, idx_in
    elif S_out is S and idx_out is not idx_in:
        raise ValueError("an update in place leaves every state where it was: S_out and idx_out have to be None")
    n_in, n_out = len(S), len(S_out)
    if S_out is S or n_out != n_in:
        _check((n_in, H, d, d), torch.float32, dev, "S", S)
        if S_out is not S:
            _check((n_out, H, d, d), torch.float32, dev, "S_out", S_out)
    else:
        _check((n_in, H, d, d), torch.float32, dev, "S S_out", S, S_out)
    if idx_in is not None and idx_out is not None:
        _check((n_seq,), torch.int32, dev, "idx_in idx_out", idx_in, idx_out)
    else:
        for idx, n, name in ((idx_in, n_in, "S"), (idx_out, n_out, "S_out")):
            if idx is not None:
                _check((n_seq,), torch.int32, dev, "index", idx)
            elif n < n_seq:
                raise ValueError(f"{name} has {n} states for {n_seq} sequences and no index")
    L = _lib.rollout()
    head = (_lib.HARTS_BF16 if dtype is torch.bfloat16 else _lib.HARTS_F32, n_seq, n_rows, H, d,
            d ** -0.5 if scale is None else scale, q.data_ptr(), k.data_ptr(), v.data_ptr(), g.data_ptr())
    tail = (_ptr(row_off), S.data_ptr(), _ptr(idx_in), n_in, S_out.data_ptr(), _ptr(idx_out), n_out, out.data_ptr())
    if kda:
        _call(dev.index, "harts_kda_step", L.harts_kda_step, *head, beta.data_ptr(), *tail)
    else:
        _call(dev.index, "harts_la_step", L.harts_la_step, *head, *tail)
    return out


def la_step(q, k, v, g, S, S_out=None, idx_in=None, idx_out=None, row_off=None, scale=None, out=None):
    """Tokens of linear attention with scalar decay, one row of q, k, v
    [rows, H, d] and g [rows, H] for each sequence, or sequence i's rows
    [row_off[i], row_off[i + 1]) one after the other.  States start from
    S[idx_in[i]] and end in S_out[idx_out[i]] (no index: i; no S_out: in
    place).  Several sequences may start from one state: a fork.  Returns o."""
    return _step(False, q, k, v, g, None, S, S_out, idx_in, idx_out, row_off, scale, out)


def kda_step(q, k, v, g, beta, S, S_out=None, idx_in=None, idx_out=None, row_off=None, scale=None, out=None):
    """The same for KDA: g [rows, H, d], beta [rows, H]."""
    return _step(True, q, k, v, g, beta, S, S_out, idx_in, idx_out, row_off, scale, out)
