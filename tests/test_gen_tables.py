"""Generation on the CPU: the host tables of harts_gen_layout / harts_gen_tables
cover every (query row, head, segment, split) exactly once, and every entry
point refuses what it documents before anything is enqueued."""
import ctypes as C
import os
import re

import numpy as np
import pytest

from oracle.gen import chain, e4m3_round, e4m3_vectors

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def L():
    from paper_2608_28158_amd import _lib
    return _lib.rollout()


def test_library_exports_every_declared_symbol(L):
    from paper_2608_28158_amd import _lib
    text = open(os.path.join(ROOT, "include", "harts_rollout.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    declared = sorted(set(re.findall(r"^\s*int\s+(harts_\w+)\s*\(", text, flags=re.M)))
    assert sorted(_lib.ROLLOUT_EXPORTS) == declared
    for name in declared:
        assert getattr(L, name).argtypes, name


def tables(L, parent, n_new, cap, Hq, Hkv):
    from paper_2608_28158_amd import _lib
    parent, n_new, cap = (np.ascontiguousarray(a, t) for a, t in
                          ((parent, np.int32), (n_new, np.int32), (cap, np.int64)))
    host = (len(parent), parent.ctypes.data, n_new.ctypes.data, cap.ctypes.data, Hq, Hkv)
    sz = _lib.GenSizes()
    _lib.check(L.harts_gen_layout(*host, C.byref(sz)), "harts_gen_layout")
    rows, order = np.zeros((sz.n_rows, 2), np.int32), np.zeros(sz.n_rows, np.int32)
    items, off = np.zeros((sz.n_items, 12), np.int32), np.zeros(sz.n_rows + 1, np.int32)
    _lib.check(L.harts_gen_tables(*host, rows.ctypes.data, order.ctypes.data, items.ctypes.data, off.ctypes.data),
               "harts_gen_tables")
    return sz, rows, order, items, off


def random_forest(rng, n):
    ids = rng.permutation(n)
    parent = np.full(n, -1, np.int32)
    for i in range(1, n):
        if rng.random() > 0.2:
            parent[ids[i]] = ids[rng.integers(max(0, i - 9), i)]
    return parent


@pytest.mark.parametrize("seed", range(24))
def test_tables_cover_every_row_and_key_once(L, seed):
    rng = np.random.default_rng(seed)
    n = int(rng.integers(1, 30))
    parent = random_forest(rng, n)
    n_new = rng.integers(0, 1 + int(rng.choice([1, 3, 200])), n)
    cap = rng.choice([0, 1, 63, 900, 5000, 70000], n)
    Hkv = int(rng.choice([1, 2, 5]))
    group = int(rng.choice([1, 3, 8]))
    sz, rows, order, items, off = tables(L, parent, n_new, cap, Hkv * group, Hkv)
    assert sz.n_rows == n_new.sum()
    want = [(s, i - n_new[s]) for s in range(n) for i in range(n_new[s])]
    assert [tuple(x) for x in rows] == want
    assert sorted(order) == list(range(sz.n_rows))
    assert sz.n_parts == off[-1] and sz.n_join == np.sum(np.diff(off) > 1)
    seen = {}
    for seg, first, row, m, split, splits, new, part, tiles, waves, _, _ in items:
        assert tiles in (1, 2) and waves in (1, 2, 4) and 0 < m <= 16 * tiles * waves and 0 <= split < splits
        assert new == n_new[seg] and row % group == 0 or m > 0
        for stacked in range(row, row + m):
            place = stacked // group
            r = order[first + place]
            s = rows[r][0]
            assert seg in chain(parent, s)
            # own rows lead the list, in order
            assert (place < new) == (s == seg)
            if s == seg:
                assert rows[r][1] + new == place
            key = (r, stacked % group, off[r] + part + split)
            assert key not in seen and off[r] <= key[2] < off[r + 1]
            seen[key] = seg
    assert len(seen) == sz.n_parts * group
    # parts run along the chain, root first
    for r in range(sz.n_rows):
        segs = [seen[(r, 0, p)] for p in range(off[r], off[r + 1])]
        assert list(dict.fromkeys(segs)) == chain(parent, rows[r][0])


@pytest.mark.parametrize("seed", range(8))
def test_items_carry_new_rows_and_divisors(L, seed):
    """Every item's own new rows, and the multiplier and shift that divide by its splits, at the edges
    of quotients up to the largest number."""
    rng = np.random.default_rng(100 + seed)
    n = int(rng.integers(1, 20))
    parent = random_forest(rng, n)
    n_new = rng.integers(0, 1 + int(rng.choice([1, 3, 200])), n)
    n_new[-1] = max(1, n_new[-1])
    cap = rng.choice([0, 1, 63, 900, 5000, 70000, 10 ** 9], n)
    _, _, _, items, _ = tables(L, parent, n_new, cap, 8, 2)
    assert len(items)
    for seg, _, _, _, _, splits, new, _, _, _, mul, shift in (map(int, x) for x in items):
        assert new == n_new[seg]
        mul &= 2 ** 32 - 1
        near = {0, 1, splits - 1, splits, splits + 1, 2 ** 31 - 1, (2 ** 31 - 1) // splits * splits}
        near |= {k * splits + e for k in (2, 3, 1000, 65536) for e in (-1, 0, 1)}
        for x in near:
            if 0 <= x < 2 ** 31:
                assert x * mul >> shift == x // splits, (x, splits)


def test_a_deep_chain_and_many_segments(L):
    n = 4000
    parent = np.arange(-1, n - 1)
    n_new = np.zeros(n, np.int32)
    n_new[-1] = 2
    sz, _, _, items, off = tables(L, parent, n_new, np.full(n, 5), 4, 2)
    assert list(off) == [0, n, 2 * n] and sz.n_items == n
    sz, *_ = tables(L, np.full(n, -1), np.ones(n, np.int32), np.full(n, 300), 16, 16)
    assert sz.n_items == n and sz.n_join == 0


def test_the_largest_capacity(L):
    """A capacity is a hint, up to the type's largest: the most splits, not none."""
    top = np.iinfo(np.int64).max
    sz, _, _, items, off = tables(L, [-1, 0], [0, 3], [top, 40], 2, 1)
    assert sz.n_items == 4097 and list(off) == [0, 4097, 2 * 4097, 3 * 4097]
    assert sorted(items[items[:, 0] == 0][:, 4]) == list(range(4096))


def test_no_rows(L):
    from paper_2608_28158_amd import _lib
    sz, rows, order, items, off = tables(L, [-1, 0], [0, 0], [10, 10], 4, 4)
    assert (sz.n_rows, sz.n_items, sz.n_parts, sz.n_join) == (0, 0, 0, 0)
    b = C.c_size_t(1)
    _lib.check(L.harts_gen_workspace_size(C.byref(sz), 4, 64, C.byref(b)), "size")
    assert b.value == 0


@pytest.mark.parametrize("parent,n_new,cap,Hq,Hkv", [
    ([1, 0], [1, 1], [1, 1], 2, 2),        # cycle
    ([0], [1], [1], 2, 2),                 # its own parent
    ([-2], [1], [1], 2, 2),
    ([1], [1], [1], 2, 2),                 # out of range
    ([-1], [-1], [1], 2, 2),
    ([-1], [1], [-1], 2, 2),
    ([-1], [1], [1], 3, 2),                # heads
    ([-1], [1], [1], 1, 2),
    ([-1], [1], [1], 0, 0),
])
def test_layout_refuses(L, parent, n_new, cap, Hq, Hkv):
    from paper_2608_28158_amd import _lib
    a = [np.ascontiguousarray(x, t) for x, t in ((parent, np.int32), (n_new, np.int32), (cap, np.int64))]
    sz = _lib.GenSizes()
    rc = L.harts_gen_layout(len(parent), a[0].ctypes.data, a[1].ctypes.data, a[2].ctypes.data, Hq, Hkv, C.byref(sz))
    assert rc == _lib.HARTS_EINVAL and _lib.last_error()


def test_layout_refuses_null_and_size(L):
    from paper_2608_28158_amd import _lib
    one, cap = np.ones(1, np.int32), np.ones(1, np.int64)
    root, sz = -one, _lib.GenSizes()
    assert L.harts_gen_layout(1, None, one.ctypes.data, cap.ctypes.data, 1, 1, C.byref(sz)) == _lib.HARTS_EINVAL
    assert L.harts_gen_layout(1, root.ctypes.data, one.ctypes.data, cap.ctypes.data, 1, 1, None) == _lib.HARTS_EINVAL
    assert L.harts_gen_layout(0, root.ctypes.data, one.ctypes.data, cap.ctypes.data, 1, 1,
                              C.byref(sz)) == _lib.HARTS_EINVAL
    many = np.full(1, 2 ** 30, np.int32)
    assert L.harts_gen_layout(1, root.ctypes.data, many.ctypes.data, cap.ctypes.data, 4, 1,
                              C.byref(sz)) == _lib.HARTS_EUNSUPPORTED


def test_layout_refuses_rows_past_64_bits(L):
    """(rows x heads, which wrapped around to a small or negative number)"""
    from paper_2608_28158_amd import _lib
    for n, heads in ((1 << 17, 65535), (1 << 18, 1 << 15)):
        root, new, cap = np.full(n, -1, np.int32), np.full(n, 2 ** 31 - 1, np.int32), np.ones(n, np.int64)
        sz = _lib.GenSizes()
        assert L.harts_gen_layout(n, root.ctypes.data, new.ctypes.data, cap.ctypes.data, heads, 1,
                                  C.byref(sz)) == _lib.HARTS_EUNSUPPORTED


# ---------------------------------------------------------------------------
# refusals of the device calls: nothing is enqueued, so any non-NULL aligned
# addresses serve as pointers
# ---------------------------------------------------------------------------
P = 1 << 20


def cache(**over):
    from paper_2608_28158_amd import _lib
    f = dict(k=P, v=2 * P, k_exp=3 * P, v_exp=4 * P, pages=5 * P, len=6 * P, n_pages=4, n_seg=2, pitch=2, H=2, d=64,
             kind=_lib.HARTS_E4M3)
    f.update(over)
    return _lib.Cache(*(f[n] for n, _ in _lib.Cache._fields_))


BAD_CACHE = [("kind", 0), ("kind", 3), ("d", 96), ("H", 0), ("H", 70000), ("n_pages", 0), ("n_seg", 0), ("pitch", 0),
             ("k", None), ("v", P + 8), ("pages", None), ("len", P + 2), ("k_exp", None), ("v_exp", P + 1)]


@pytest.mark.parametrize("field,value", BAD_CACHE)
def test_cache_calls_refuse_a_bad_cache(L, field, value):
    from paper_2608_28158_amd import _lib
    c = cache(**{field: value})
    for fn in (L.harts_cache_write, L.harts_cache_read):
        assert fn(C.byref(c), P, 1, P, P, None) in (_lib.HARTS_EINVAL, _lib.HARTS_EUNSUPPORTED)
    sz = _lib.GenSizes(1, 1, 1, 0)
    assert L.harts_gen_attn(C.byref(c), C.byref(sz), P, P, P, 2, 1.0, 7 * P, 8 * P, None, None, 0,
                            None) in (_lib.HARTS_EINVAL, _lib.HARTS_EUNSUPPORTED)


def test_cache_calls_refuse_rows(L):
    from paper_2608_28158_amd import _lib
    c = C.byref(cache())
    for fn in (L.harts_cache_write, L.harts_cache_read):
        assert fn(None, P, 1, P, P, None) == _lib.HARTS_EINVAL
        assert fn(c, P, -1, P, P, None) == _lib.HARTS_EINVAL
        assert fn(c, None, 1, P, P, None) == _lib.HARTS_EINVAL
        assert fn(c, P, 1, None, P, None) == _lib.HARTS_EINVAL
        assert fn(c, P, 1, P, P + 4, None) == _lib.HARTS_EINVAL
        assert fn(c, P, 1 << 40, P, P, None) == _lib.HARTS_EUNSUPPORTED
        assert fn(c, None, 0, None, None, None) == _lib.HARTS_OK


def test_attention_refuses(L):
    from paper_2608_28158_amd import _lib
    def call(sizes=(4, 4, 8, 4), Hq=4, q=7 * P, o=8 * P, lse=9 * P, ws=10 * P, ws_bytes=8 * 4 * 66 * 4, items=P):
        sz = _lib.GenSizes(*sizes)
        return L.harts_gen_attn(C.byref(cache()), C.byref(sz), items, P, P, Hq, 1.0, q, o, lse, ws, ws_bytes, None)
    E, U = _lib.HARTS_EINVAL, _lib.HARTS_EUNSUPPORTED
    assert call(Hq=3) == U and call(Hq=1) == U and call(Hq=1 << 17) == U
    assert call(q=None) == E and call(o=8 * P + 8) == E and call(items=None) == E
    assert call(ws=None) == E and call(ws_bytes=8 * 4 * 66 * 4 - 1) == E
    assert call(o=7 * P) == E and call(o=7 * P + 16) == E         # o over q
    assert call(sizes=(2 ** 62, 4, 8, 4)) == E and call(sizes=(4, 2 ** 62, 8, 4)) == E
    assert call(sizes=(-1, 4, 8, 4)) == E and call(sizes=(4, 0, 8, 4)) == E and call(sizes=(2 ** 40, 1, 1, 0)) == E
    assert call(sizes=(0, 0, 0, 0), q=None) == _lib.HARTS_OK


def test_steps_refuse(L):
    from paper_2608_28158_amd import _lib
    E, U = _lib.HARTS_EINVAL, _lib.HARTS_EUNSUPPORTED
    def call(kda, dtype=_lib.HARTS_BF16, n_seq=2, n_rows=2, H=2, d=64, q=P, o=5 * P, off=None, S=16 * P, ii=None, n_in=2,
             So=32 * P, io=None, n_out=2, beta=6 * P):
        head = (dtype, n_seq, n_rows, H, d, 1.0, q, 2 * P, 3 * P, 4 * P)
        tail = (off, S, ii, n_in, So, io, n_out, o, None)
        return L.harts_kda_step(*head, beta, *tail) if kda else L.harts_la_step(*head, *tail)
    for kda in (False, True):
        assert call(kda, dtype=2) == U and call(kda, d=32) == U and call(kda, H=0) == U
        assert call(kda, n_seq=-1) == E and call(kda, n_rows=1) == E and call(kda, n_in=-1) == E
        assert call(kda, q=None) == E and call(kda, o=None) == E and call(kda, S=None) == E and call(kda, So=None) == E
        assert call(kda, q=P + 8) == E and call(kda, S=16 * P + 4) == E
        assert call(kda, o=P) == E and call(kda, o=3 * P + 16) == E                # o over an input
        assert call(kda, o=4 * P) == E and call(kda, o=16 * P) == E and call(kda, o=32 * P) == E
        assert call(kda, So=2 * P) == E and call(kda, So=4 * P) == E               # S_out over k, g
        assert call(kda, So=16 * P, ii=P, io=2 * P) == E                           # in place, two indexes
        assert call(kda, So=16 * P, n_out=1) == E                                  # in place, two sizes
        assert call(kda, So=16 * P + 16) == E                                      # overlap
        assert call(kda, n_seq=0, q=None) == _lib.HARTS_OK
        assert call(kda, n_in=2 ** 62) == U and call(kda, n_seq=2 ** 40, n_rows=2 ** 40) == U
    assert call(True, beta=None) == E


def test_outputs_over_other_arguments_are_refused(L):
    """Every output of every call over every other argument, at its first bytes and at its last."""
    from paper_2608_28158_amd import _lib
    H, d, n = 2, 64, 3
    held, table = {_lib.HARTS_BF16: 4 * H * 64 * d * 2, _lib.HARTS_E4M3: 4 * H * 64 * d}, 2 * 2 * 4
    def refused(fn, sizes, written, aliasable=()):
        at = {name: (20 + 10 * i) * P for i, name in enumerate(sizes)}
        assert max(sizes.values()) < 10 * P
        for w in written:
            for other in sizes:
                if other == w or (w, other) in aliasable:
                    continue
                for place in (at[other], at[other] + (sizes[other] - 1) // 16 * 16, at[other] - (sizes[w] - 1) // 16 * 16):
                    assert fn({**at, w: place}) == _lib.HARTS_EINVAL, (w, other)
                    assert "overlap" in _lib.last_error(), (w, other, _lib.last_error())

    for kind in (_lib.HARTS_BF16, _lib.HARTS_E4M3):
        parts = dict(k=held[kind], v=held[kind], pages=table, len=2 * 4)
        if kind == _lib.HARTS_E4M3:
            parts.update(k_exp=4 * H * 64, v_exp=4 * H * 64)
        cached = [x for x in ("k", "v", "k_exp", "v_exp") if x in parts]
        def of(at):
            return cache(**{x: at.get(x) for x in ("k", "v", "k_exp", "v_exp", "pages", "len")}, kind=kind, H=H, d=d)
        rows = dict(rows=n * 8, k_new=n * H * d * 2, v_new=n * H * d * 2)
        refused(lambda at: L.harts_cache_write(C.byref(of(at)), at["rows"], n, at["k_new"], at["v_new"], None),
                {**parts, **rows}, cached)
        refused(lambda at: L.harts_cache_read(C.byref(of(at)), at["rows"], n, at["k_new"], at["v_new"], None),
                {**parts, **rows}, ["k_new", "v_new"])
        sz = _lib.GenSizes(n, 5, 8, 2)
        ws = 8 * 4 * (d + 2) * 4
        refused(lambda at: L.harts_gen_attn(C.byref(of(at)), C.byref(sz), at["items"], at["order"], at["off"], 4, 1.0,
                                            at["q"], at["o"], at["lse"], at["ws"], ws, None),
                {**parts, "items": 5 * 48, "order": n * 4, "off": (n + 1) * 4, "q": n * 4 * d * 2, "o": n * 4 * d * 2,
                 "lse": n * 4 * 4, "ws": ws}, ["o", "lse", "ws"])
    for kda in (False, True):
        state = H * d * d * 4
        x = dict(q=n * H * d * 2, k=n * H * d * 2, v=n * H * d * 2, g=n * H * 4 * (d if kda else 1), off=3 * 4, S=2 * state,
                 ii=2 * 4, So=2 * state, io=2 * 4, o=n * H * d * 2)
        if kda:
            x["beta"] = n * H * 4
        def step(at):
            head = (_lib.HARTS_BF16, 2, n, H, d, 1.0, at["q"], at["k"], at["v"], at["g"])
            tail = (at["off"], at["S"], at["ii"], 2, at["So"], at["io"], 2, at["o"], None)
            return L.harts_kda_step(*head, at["beta"], *tail) if kda else L.harts_la_step(*head, *tail)
        refused(step, x, ["o", "So"])


def test_gates_of_linear_attention_have_float_alignment(L):
    """g [n_rows][H] is read one by one; only what comes after the alignment is refused here (o over k)."""
    from paper_2608_28158_amd import _lib
    def call(g, kda):
        head = (_lib.HARTS_BF16, 2, 2, 5, 64, 1.0, P, 2 * P, 3 * P, g)
        tail = (None, 16 * P, None, 2, 32 * P, None, 2, 2 * P, None)
        rc = L.harts_kda_step(*head, 6 * P, *tail) if kda else L.harts_la_step(*head, *tail)
        return rc, _lib.last_error()
    for g in (4 * P + 4, 4 * P + 20, 4 * P + 8):
        assert call(g, False) == (_lib.HARTS_EINVAL, "harts_la_step: o overlaps an input")
        assert call(g, True) == (_lib.HARTS_EINVAL, "harts_kda_step: misaligned pointer")
    assert call(4 * P + 2, False) == (_lib.HARTS_EINVAL, "harts_la_step: misaligned pointer")


def test_python_calls_refuse_tensors_of_the_cpu(L):
    import torch
    from paper_2608_28158_amd.rollout import RolloutCache, kda_step, la_step
    x, g, S = torch.zeros(1, 2, 64), torch.zeros(1, 2), torch.zeros(1, 2, 64, 64)
    with pytest.raises(RuntimeError, match="GPU only"):
        la_step(x, x, x, g, S)
    with pytest.raises(RuntimeError, match="GPU only"):
        kda_step(x, x, x, x, g, S)
    with pytest.raises(ValueError, match="float32 or bfloat16"):
        la_step(x.double(), x, x, g, S)
    with pytest.raises(ValueError, match="float32 or bfloat16"):
        la_step(x[0], x, x, g, S)
    with pytest.raises(TypeError):
        la_step(None, x, x, g, S)
    with pytest.raises(RuntimeError, match="GPU only"):
        RolloutCache(2, 2, 1, 2, 64, device="cpu")


def test_sizes_past_32_bits_are_refused(L):
    from paper_2608_28158_amd import _lib
    from paper_2608_28158_amd.rollout import RolloutCache
    b = C.c_size_t()
    for parts, heads in ((2 ** 31, 4), (2 ** 62, 4), (8, 65536), (8, 2 ** 30)):
        assert L.harts_gen_workspace_size(C.byref(_lib.GenSizes(4, 4, parts, 4)), heads, 64, C.byref(b)) == _lib.HARTS_EINVAL
    assert L.harts_gen_workspace_size(C.byref(_lib.GenSizes(4, 4, 2 ** 31 - 1, 4)), 65535, 128, C.byref(b)) == _lib.HARTS_OK
    assert b.value == (2 ** 31 - 1) * 65535 * 130 * 4
    for over in (dict(n_pages=2 ** 32 + 1), dict(n_seg=2 ** 31), dict(pitch=2 ** 32 + 1), dict(heads=65536)):
        with pytest.raises(ValueError, match="at most"):
            RolloutCache(**{**dict(n_pages=1, n_seg=1, pitch=1, heads=1, d=64), **over})


def test_host_tables_are_not_cut_to_size():
    """Numbers that the tables' types do not hold are refused, not wrapped around or cut off."""
    import torch
    from paper_2608_28158_amd.rollout import _host_table
    for good in ([-1, 0, 7], np.array([-1, 0, 7], np.int64), np.array([-1.0, 0.0, 7.0]), torch.tensor([-1, 0, 7])):
        a = _host_table("parent", good, 3, np.int32)
        assert a.dtype == np.int32 and a.flags.c_contiguous and list(a) == [-1, 0, 7]
    assert list(_host_table("n_new", np.arange(6)[::2], 3, np.int32)) == [0, 2, 4]
    assert _host_table("capacity", [2 ** 63 - 1], 1, np.int64)[0] == 2 ** 63 - 1
    for bad in (np.array([2 ** 32 + 1]), np.array([-2 ** 32]), [1.5], [float("nan")], np.array([2 ** 31]), [1e300]):
        with pytest.raises(ValueError, match="whole numbers of int32"):
            _host_table("n_new", bad, 1, np.int32)
    with pytest.raises(ValueError, match="whole numbers of int64"):
        _host_table("capacity", np.array([2 ** 64 - 1], np.uint64), 1, np.int64)
    for shape in ([1], [1, 2, 3], [[1, 2]], 1):
        with pytest.raises(ValueError, match="one entry for each"):
            _host_table("n_new", shape, 2, np.int32)


# ---------------------------------------------------------------------------
# the oracle's rounding, against every code
# ---------------------------------------------------------------------------

def test_e4m3_rounding_against_the_codes():
    codes = np.array([(1 if s == 0 else -1) * (2.0 ** -9 * m if e == 0 else 2.0 ** (e - 7) * (1 + m / 8))
                      for s in (0, 1) for e in range(16) for m in range(8) if not (e == 15 and m == 7)])
    assert np.array_equal(e4m3_round(codes), codes)
    pos = np.unique(np.abs(codes))
    mid = (pos[1:] + pos[:-1]) / 2
    even = np.where((np.arange(len(mid)) % 2) == 0, pos[:-1], pos[1:])    # codes alternate in parity from 0
    assert np.array_equal(e4m3_round(mid), even)
    assert np.array_equal(e4m3_round(np.nextafter(mid, 0)), pos[:-1])
    assert np.array_equal(e4m3_round(np.nextafter(mid, 1e9)), pos[1:])


def test_e4m3_scales():
    x = np.array([[448.0, 1], [449.0, 1], [0.0, 0], [1.75, -0.3], [1.7501, 0], [2.0 ** -133, 0], [np.inf, 3.0]])
    v, e = e4m3_vectors(x)
    assert list(e) == [0, 1, -126, -8, -7, -126, -7]
    assert v[0, 0] == 448 and np.isnan(v[6, 0]) and v[6, 1] == 3.0 and v[5, 0] == 2.0 ** -133
