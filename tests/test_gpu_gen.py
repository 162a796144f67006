"""The paged cache and attention over a forest of cached segments on the GPU,
against the float64 oracle.

Tolerances, per output.  The operands are bf16 values in both, products are
summed in float32; weights are rounded to bf16 for the second product (half a
step, 2^-8 of each), so o may be off by 2^-8 of the weighted sum of |v| and by
its own rounding, 2^-8 of o.  A score of d products is off by at most
(d + 4) 2^-24 of the sum of |q||k| (float32 sums and the scaling), a weight by
that relative amount twice (itself and the sum), the same for lse absolutely;
exponentials, logarithms and joins add a few float32 steps (2^-20 in all).
What the cache stands for is exact."""
import numpy as np
import pytest
import torch

from oracle.gen import e4m3_vectors, forest_decode

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")


def bf16_values(x):
    return torch.from_numpy(np.asarray(x, np.float32)).to(torch.bfloat16)


def f64(t):
    return t.detach().cpu().double().numpy()


def new_cache(n_pages, n_seg, pitch, H, d, kind, layers=1):
    """A cache whose unused cells hold NaN and infinities."""
    from paper_2608_28158_amd.rollout import RolloutCache
    c = RolloutCache(n_pages, n_seg, pitch, H, d, kind=kind, layers=layers)
    if kind == "bf16":
        c.k.fill_(float("nan"))
        c.v.fill_(float("inf"))
    else:
        c.k.view(torch.uint8).fill_(0x7f)
        c.v.view(torch.uint8).fill_(0xff)
        c.k_exp.fill_(254)
        c.v_exp.fill_(254)
    return c


def table(rows):
    return torch.tensor(rows, dtype=torch.int32).reshape(-1, 2).cuda()


def stands_for(x, kind):
    return f64(x) if kind == "bf16" else e4m3_vectors(f64(x))[0]


# ---------------------------------------------------------------------------
# cache
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("H,d", [(1, 64), (3, 128), (16, 128), (20, 64)])
@pytest.mark.parametrize("lens", [[1], [63, 64, 65], [200, 1, 129]])
def test_written_rows_read_back(kind, H, d, lens):
    rng = np.random.default_rng(len(lens) * d + H)
    pitch = -(-max(lens) // 64)
    c = new_cache(3 * pitch + 2, 3, pitch, H, d, kind, layers=2)
    for s, n in enumerate(lens):
        c.reserve(s, n)
        c.len[s] = n
    rows = [(s, p) for s, n in enumerate(lens) for p in range(n)]
    rng.shuffle(rows)
    # magnitudes over the whole range of bf16, zeros, vectors of zeros
    x = [rng.standard_normal((len(rows), H, d)) * 2.0 ** rng.integers(-136, 120, (len(rows), H, 1)) for _ in range(2)]
    x[0][:, :, ::7] = 0
    x[1][0] = 0
    k, v = (bf16_values(a) for a in x)
    before = [t.clone() for t in (c.k, c.v)]
    c.write(table(rows), k.cuda(), v.cuda(), layer=1)
    ends = [(s, p - lens[s]) for s, p in rows]               # counted from the end
    kb, vb = c.read(table(ends), layer=1)
    assert np.array_equal(f64(kb), stands_for(k, kind)) and np.array_equal(f64(vb), stands_for(v, kind))
    assert torch.equal(c.k[0].view(torch.uint8), before[0][0].view(torch.uint8))      # the other layer
    # cells behind the segments' ends
    for s, n in enumerate(lens):
        if n % 64:
            page = int(c.pages[s, n // 64])
            for t, b in ((c.k, before[0]), (c.v, before[1])):
                assert torch.equal(t[1, page, :, n % 64:].view(torch.uint8), b[1, page, :, n % 64:].view(torch.uint8))


@pytest.mark.parametrize("d", [64, 128])
def test_e4m3_of_special_values(d):
    x = np.zeros((6, 1, d))
    x[0, 0, :4] = [np.inf, 1.0, -np.inf, 448.0]
    x[1, 0, :3] = [np.nan, -3.0, 0.1]
    x[2, 0, :3] = [449.0, 448.0, -1.0]
    x[3, 0, :2] = [2.0 ** -133, -2.0 ** -132]
    x[4] = np.inf
    x[5, 0, :] = np.linspace(-448, 448, d)
    c = new_cache(1, 1, 1, 1, d, "e4m3")
    c.reserve(0, 6)
    c.len[0] = 6
    b = bf16_values(x)
    c.write(table([(0, i) for i in range(6)]), b.cuda(), b.flip(0).cuda())
    k, v = c.read(table([(0, i) for i in range(6)]))
    want, e = e4m3_vectors(f64(b))
    assert np.array_equal(f64(k), want, equal_nan=True) and np.array_equal(f64(v)[::-1], want, equal_nan=True)
    page = int(c.pages[0, 0])
    assert np.array_equal(c.k_exp[0, page, :, :6].cpu().numpy().T.astype(int), e + 127)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_entries_that_name_no_row(kind):
    c = new_cache(4, 3, 2, 2, 64, kind)
    c.reserve(0, 100)
    c.len[0] = 100
    c.len[1] = 70                                            # rows, but no pages
    c.reserve(2, 128)
    c.len[2] = 500                                           # more than the table holds
    c.pages[2, 1] = 77                                       # a page that does not exist
    good = [(0, 99), (0, -100), (2, 63), (2, -437)]          # 500 - 437 = row 63 again
    bad = [(0, 100), (0, -101), (1, 5), (1, 69), (2, 64), (2, 127), (2, 128), (2, -1), (-1, 0), (3, 0), (0, 2 ** 31 - 1),
           (0, -2 ** 31)]
    x = bf16_values(np.random.default_rng(0).standard_normal((len(bad) + 3, 2, 64))).cuda()
    before = [t.clone().view(torch.uint8) for t in (c.k, c.v)]
    c.write(table(bad), x[:len(bad)], x[:len(bad)])
    assert torch.equal(c.k.view(torch.uint8), before[0]) and torch.equal(c.v.view(torch.uint8), before[1])
    c.write(table(good[:3]), x[-3:], x[-3:])
    k, v = c.read(table(good + bad))
    assert np.array_equal(f64(k[:3]), stands_for(x[-3:], kind)) and torch.equal(k[3], k[2])
    assert not f64(k[4:]).any() and not f64(v[4:]).any()


def test_pages_are_handed_out_and_taken_back():
    c = new_cache(5, 3, 4, 1, 64, "bf16")
    c.reserve(0, 130)
    c.reserve(0, 100)
    c.reserve(1, 1)
    assert c.free_pages == 1
    used = c.pages[0, :3].tolist() + c.pages[1, :1].tolist()
    assert sorted(set(used)) == sorted(used) and min(used) >= 0 and int(c.pages[0, 3]) == -1
    with pytest.raises(RuntimeError):
        c.reserve(2, 65)
    with pytest.raises(ValueError):
        c.reserve(2, 257)
    with pytest.raises(ValueError):
        c.reserve(3, 1)
    assert c.free_pages == 1
    c.release(0)
    assert c.free_pages == 4 and int(c.pages[0].max()) == -1
    c.reserve(2, 256)


def test_no_rows_at_all():
    from paper_2608_28158_amd.rollout import RolloutBatch
    c = new_cache(1, 1, 1, 2, 64, "bf16")
    e = torch.empty((0, 2, 64), dtype=torch.bfloat16, device="cuda")
    c.write(torch.empty((0, 2), dtype=torch.int32, device="cuda"), e, e)
    assert c.read(torch.empty((0, 2), dtype=torch.int32, device="cuda"))[0].shape == (0, 2, 64)
    o, lse = RolloutBatch(c, [-1], [0], 4).attend(torch.empty((0, 4, 64), dtype=torch.bfloat16, device="cuda"))
    assert o.shape == (0, 4, 64) and lse.shape == (0, 4)


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------

def filled(parent, lens, Hkv, d, kind, rng, spread=1.0):
    """A cache with the segments' rows, and what they stand for."""
    n = len(parent)
    pitch = max(1, -(-max(lens) // 64)) + 1
    c = new_cache(sum(-(-x // 64) for x in lens) + 1, n, pitch, Hkv, d, kind)
    order = rng.permutation(n)
    K, V = [None] * n, [None] * n
    for s in order:
        c.reserve(int(s), lens[s])
        c.len[int(s)] = lens[s]
        k, v = (bf16_values(spread * rng.standard_normal((lens[s], Hkv, d))) for _ in range(2))
        if lens[s]:
            c.write(table([(s, p) for p in range(lens[s])]), k.cuda(), v.cuda())
        K[s], V[s] = stands_for(k, kind), stands_for(v, kind)
    return c, K, V


def bounds(o, mag, reach, lse, d):
    z = (d + 4) * 2.0 ** -24 * reach
    tol_o = 2.0 ** -8 * (np.abs(o) + mag) + (2 * z[..., None] + 2.0 ** -20) * mag
    tol_lse = z + 2.0 ** -20 * (1 + np.abs(np.where(np.isfinite(lse), lse, 0)))
    return tol_o, tol_lse


def compare(o, lse, ref, d):
    ro, rl, mag, reach = ref
    tol_o, tol_l = bounds(ro, mag, reach, rl, d)
    got, gl = f64(o), f64(lse)
    assert np.all(np.isfinite(got))
    some = np.isfinite(rl)
    assert np.all(gl[~some] == -np.inf) and not got[~some].any()
    assert np.all(np.abs(got - ro) <= tol_o), np.max(np.abs(got - ro) / np.maximum(tol_o, 1e-30))
    assert np.all(np.abs(gl[some] - rl[some]) <= tol_l[some]), np.max(np.abs(gl[some] - rl[some]) / tol_l[some])


# parents, rows, new rows
FORESTS = {
    "one_token": ([-1], [1], [1]),
    "page_edges": ([-1] * 5, [63, 64, 65, 128, 129], [1, 1, 2, 1, 3]),
    "two_samples": ([-1, 0, 0], [100, 1, 33], [0, 1, 1]),
    "long_prefix": ([-1] + [0] * 9, [2500] + [1, 64, 7, 200, 31, 33, 65, 128, 96], [0] + [1] * 9),
    "short_prefix": ([-1] + [0] * 9, [300] + [1, 64, 7, 200, 31, 33, 65, 128, 96], [0] + [1] * 9),
    "forest_any_order": ([3, 3, -1, -1, 0, 0, 1, 2], [40, 65, 500, 130, 9, 1, 70, 5], [0, 2, 1, 3, 9, 1, 4, 5]),
    "empty_segments": ([-1, 0, 1, 1, -1], [0, 70, 0, 3, 0], [0, 0, 0, 2, 0]),
    "rows_seeing_nothing": ([-1, -1, 1], [2, 0, 1], [5, 2, 3]),
    "prompt": ([-1], [300], [300]),
    "prompt_continued": ([-1, 0], [450, 210], [0, 150]),
    "many_short": ([-1] * 40, list(range(1, 41)), [1] * 40),
    "deep": ([-1, 0, 1, 2, 3, 4, 5, 6], [1, 90, 2, 64, 3, 5, 32, 31], [0, 1, 0, 0, 2, 0, 0, 4]),
}
HEADS = [(4, 4, 64), (8, 2, 128), (6, 1, 64), (3, 3, 128), (16, 1, 128)]


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("Hq,Hkv,d", HEADS)
@pytest.mark.parametrize("name", FORESTS)
def test_forests(name, Hq, Hkv, d, kind):
    from paper_2608_28158_amd.rollout import RolloutBatch
    parent, lens, new = FORESTS[name]
    rng = np.random.default_rng(sum(lens) + Hq + d)
    c, K, V = filled(parent, lens, Hkv, d, kind, rng)
    q = bf16_values(rng.standard_normal((sum(new), Hq, d)))
    batch = RolloutBatch(c, parent, new, Hq, capacity=lens if Hq != 6 else None)
    out = torch.full((sum(new), Hq, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    o, lse = batch.attend(q.cuda(), out=out)
    assert o is out
    compare(o, lse, forest_decode(parent, new, K, V, f64(q), d ** -0.5), d)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("seed", range(6))
def test_random_forests(seed, kind):
    from paper_2608_28158_amd.rollout import RolloutBatch
    rng = np.random.default_rng(900 + seed)
    n = int(rng.integers(2, 14))
    parent = [-1] + [int(rng.integers(-1, i)) for i in range(1, n)]
    lens = [int(x) for x in rng.choice([0, 1, 5, 32, 64, 97, 500, 1100], n)]
    new = [int(min(x, rng.choice([0, 1, 2, 40]))) for x in lens]
    new[-1] = 1
    Hq, Hkv, d = HEADS[seed % len(HEADS)]
    c, K, V = filled(parent, lens, Hkv, d, kind, rng, spread=float(rng.choice([0.1, 1, 3])))
    q = bf16_values(rng.standard_normal((sum(new), Hq, d)))
    cap = [int(x) for x in rng.choice([0, 300, 100000], n)]          # a hint, right or wrong
    scale = float(rng.choice([-0.1, 0.0, 0.3]))
    o, lse = RolloutBatch(c, parent, new, Hq, capacity=cap).attend(q.cuda(), scale=scale)
    compare(o, lse, forest_decode(parent, new, K, V, f64(q), scale), d)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_a_long_shared_prefix(kind):
    """33 samples of a 20,000-row prefix: several splits, tiles of 128 rows, rows of many parts."""
    from paper_2608_28158_amd.rollout import RolloutBatch
    rng = np.random.default_rng(5)
    parent, lens, new = [-1] + [0] * 33, [20011] + [int(x) for x in rng.integers(1, 300, 33)], [0] + [1] * 33
    c, K, V = filled(parent, lens, 2, 128, kind, rng)
    q = bf16_values(rng.standard_normal((33, 8, 128)))
    o, lse = RolloutBatch(c, parent, new, 8, capacity=lens).attend(q.cuda())
    compare(o, lse, forest_decode(parent, new, K, V, f64(q), 128 ** -0.5), 128)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_hidden_rows_that_are_not_finite(kind, d):
    """A drafted row's NaN or infinity reaches its own and later rows only."""
    from paper_2608_28158_amd.rollout import RolloutBatch
    rng = np.random.default_rng(8)
    parent, lens, new = [-1, 0, 0], [70, 40, 66], [0, 20, 35]
    c, K, V = filled(parent, lens, 2, d, kind, rng)
    q = bf16_values(rng.standard_normal((55, 4, d)))
    ref = forest_decode(parent, new, K, V, f64(q), d ** -0.5)
    batch = RolloutBatch(c, parent, new, 4, capacity=lens)
    rows = [(1, 25), (1, 38), (2, 60)]                      # new rows 5, 18 and (of the other) 29
    for bad in (float("nan"), float("inf")):
        k, v = c.read(table(rows))
        k[:] = bad
        v[:, 1, 3:9] = bad
        c.write(table(rows), k, v)
        o, lse = batch.attend(q.cuda())
        clean = np.r_[0:5, 20:49]
        compare(o[clean], lse[clean], [x[clean] for x in ref], d)
        hit = np.r_[5:20, 49:55]
        assert np.all(np.isnan(f64(o[hit])[:, 2:, 3:9]))


def test_scores_of_minus_infinity_and_large_scores():
    from paper_2608_28158_amd.rollout import RolloutBatch
    rng = np.random.default_rng(3)
    parent, lens, new = [-1, 0], [300, 40], [0, 1]
    c, K, V = filled(parent, lens, 1, 64, "bf16", rng, spread=30.0)      # scores of several hundred
    q = bf16_values(30 * rng.standard_normal((1, 2, 64)))
    batch = RolloutBatch(c, parent, new, 2, capacity=lens)
    compare(*batch.attend(q.cuda()), forest_decode(parent, new, K, V, f64(q), 0.125), 64)
    # every key at minus infinity: a row without weight
    k, v = (torch.zeros((340, 1, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    k[:, 0, 0] = float("-inf")
    v[:] = 1
    c.write(table([(0, p) for p in range(300)] + [(1, p) for p in range(40)]), k, v)
    one = torch.zeros((1, 2, 64), dtype=torch.bfloat16, device="cuda")
    one[:, :, 0] = 1
    o, lse = batch.attend(one)
    assert not f64(o).any() and np.all(f64(lse) == -np.inf)
    k[5, 0, 0] = 0
    c.write(table([(0, 5)]), k[5:6], v[5:6])
    o, lse = batch.attend(one)
    assert np.all(f64(o) == 1) and not f64(lse).any()


def test_pages_that_do_not_exist_hold_no_keys():
    from paper_2608_28158_amd.rollout import RolloutBatch
    rng = np.random.default_rng(4)
    c, K, V = filled([-1], [250], 2, 64, "bf16", rng)
    q = bf16_values(rng.standard_normal((1, 4, 64)))
    c.pages[0, 1] = -1
    c.pages[0, 3] = 10 ** 6
    o, lse = RolloutBatch(c, [-1], [1], 4).attend(q.cuda())
    keep = np.r_[0:64, 128:192]
    compare(o, lse, forest_decode([-1], [1], [K[0][keep]], [V[0][keep]], f64(q), 0.125), 64)
    c.pages[0, 4:] = -1
    c.len[0] = 10 ** 9                                       # more rows than the table has: the query sees them all
    o2, _ = RolloutBatch(c, [-1], [1], 4).attend(q.cuda())
    assert torch.equal(o2, o)
    c.len[0] = -5
    o3, l3 = RolloutBatch(c, [-1], [1], 4).attend(q.cuda())
    assert not f64(o3).any() and np.all(f64(l3) == -np.inf)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_offsets_past_32_bits(kind):
    """Pages whose first element lies past 2^32 bytes and 2^31 elements, and one far below."""
    from paper_2608_28158_amd.rollout import RolloutBatch, RolloutCache
    rng = np.random.default_rng(7)
    H, d, n_pages = 40, 128, 13500
    assert (n_pages - 10) * H * 64 * d > 2 ** 32
    c = RolloutCache(n_pages, 2, 3, H, d, kind=kind)
    lens = [150, 70]
    c.pages[0] = torch.tensor([n_pages - 1, 4, n_pages - 3], dtype=torch.int32)
    c.pages[1, :2] = torch.tensor([n_pages - 2, 0], dtype=torch.int32)
    c.len.copy_(torch.tensor(lens, dtype=torch.int32))
    K, V = [], []
    for s, n in enumerate(lens):
        k, v = (bf16_values(rng.standard_normal((n, H, d))) for _ in range(2))
        rows = table([(s, p) for p in range(n)])
        c.write(rows, k.cuda(), v.cuda())
        K.append(stands_for(k, kind))
        V.append(stands_for(v, kind))
        kb, vb = c.read(rows)
        assert np.array_equal(f64(kb), K[s]) and np.array_equal(f64(vb), V[s])
    for new in ([0, 1], [0, 70]):                            # few rows, and a tile of many
        q = bf16_values(rng.standard_normal((sum(new), H, d)))
        o, lse = RolloutBatch(c, [-1, 0], new, H, capacity=lens).attend(q.cuda())
        compare(o, lse, forest_decode([-1, 0], new, K, V, f64(q), d ** -0.5), d)


def test_runs_are_bitwise_equal():
    from paper_2608_28158_amd.rollout import RolloutBatch
    rng = np.random.default_rng(6)
    parent, lens, new = FORESTS["long_prefix"]
    c, _, _ = filled(parent, lens, 2, 128, "e4m3", rng)
    q = bf16_values(rng.standard_normal((9, 8, 128))).cuda()
    batch = RolloutBatch(c, parent, new, 8)
    first = batch.attend(q)
    for _ in range(3):
        again = batch.attend(q)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


# ---------------------------------------------------------------------------
# as a program uses them
# ---------------------------------------------------------------------------

def test_generation_by_graph_replay():
    """Two layers; each step is one replay: lengths grow, rows are written, queries attend.  Every
    replay is checked against an eager pass over a cache of its own, and the last against the oracle."""
    from paper_2608_28158_amd.rollout import RolloutBatch
    rng = np.random.default_rng(11)
    parent, lens, new = [-1, 0, 0, 0], [90, 60, 63, 1], [0, 1, 1, 2]
    caches, rows0 = [], [90, 61, 64, 3]
    K = [[None] * 4 for _ in range(2)]
    V = [[None] * 4 for _ in range(2)]
    for _ in range(2):
        c = new_cache(12, 4, 3, 2, 64, "e4m3", layers=2)
        for s, n in enumerate(lens):
            c.reserve(s, n + 40)
            c.len[s] = n
        caches.append(c)
    for layer in range(2):
        for s, n in enumerate(lens):
            k, v = (bf16_values(rng.standard_normal((n, 2, 64))) for _ in range(2))
            K[layer][s], V[layer][s] = stands_for(k, "e4m3"), stands_for(v, "e4m3")
            for c in caches:
                c.write(table([(s, p) for p in range(n)]), k.cuda(), v.cuda(), layer)
    batch = [RolloutBatch(c, parent, new, 4) for c in caches]
    n = batch[0].n_rows
    buf = {x: torch.zeros((2, n, 4 if x == "q" else 2, 64), dtype=torch.bfloat16, device="cuda") for x in "qkv"}
    out = torch.zeros((2, n, 4, 64), dtype=torch.bfloat16, device="cuda")

    def step(b, o):
        b.advance()
        return [(b.write(buf["k"][i], buf["v"][i], i), b.attend(buf["q"][i], i, out=o[i]))[1] for i in range(2)]

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(batch[0], out)
    assert rows0[0] == lens[0] and caches[0].len.tolist() == lens         # captured, not run
    eager = torch.zeros_like(out)
    for t in range(5):
        fresh = {x: bf16_values(rng.standard_normal(tuple(buf[x].shape))) for x in "qkv"}
        for x in "qkv":
            buf[x].copy_(fresh[x])
        graph.replay()
        step(batch[1], eager)
        torch.cuda.synchronize()
        assert torch.equal(out, eager) and torch.equal(caches[0].len, caches[1].len)
        for i in range(2):
            ks, vs = stands_for(fresh["k"][i], "e4m3"), stands_for(fresh["v"][i], "e4m3")
            for j, (s, _) in enumerate(batch[0].rows.tolist()):
                K[i][s] = np.concatenate([K[i][s], ks[j:j + 1]])
                V[i][s] = np.concatenate([V[i][s], vs[j:j + 1]])
            ref = forest_decode(parent, new, K[i], V[i], f64(fresh["q"][i]), 0.125)
            compare(out[i], torch.from_numpy(ref[1]), ref, 64)


def test_streams_and_two_graphs_of_one_batch():
    from paper_2608_28158_amd.rollout import RolloutBatch
    rng = np.random.default_rng(12)
    parent, lens, new = FORESTS["long_prefix"]
    c, K, V = filled(parent, lens, 2, 64, "bf16", rng)
    batch = RolloutBatch(c, parent, new, 4)
    qs = [bf16_values(rng.standard_normal((9, 4, 64))).cuda() for _ in range(2)]
    want = [batch.attend(q)[0].clone() for q in qs]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = batch.attend(qs[1])[0]
    other = batch.attend(qs[0])[0]
    torch.cuda.synchronize()
    assert torch.equal(got, want[1]) and torch.equal(other, want[0])
    graphs, outs = [], []
    for q in qs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(batch.attend(q)[0])
        graphs.append(g)
    for _ in range(3):
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graphs[1].replay()
        graphs[0].replay()
        batch.attend(qs[0])
        torch.cuda.synchronize()
        assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1])


def test_generated_rows_agree_with_the_training_attention():
    """Rows generated one at a time through the cache give the outputs that the
    packed training attention gives for the finished tree: each within its
    bound of the exact one, so within the sum of both."""
    from oracle.attn import forest_attention
    from paper_2608_28158_amd.rollout import RolloutBatch
    rng = np.random.default_rng(13)
    parent, lens = [-1, 0, 0, 1], [70, 30, 20, 25]
    H, d, C = 2, 64, sum(lens)
    first = np.concatenate([[0], np.cumsum(lens)])
    q, k, v = (bf16_values(rng.standard_normal((C, H, d))) for _ in range(3))
    ref = forest_attention(np.array(parent), np.array(lens), f64(q), f64(k), f64(v), d ** -0.5)["o"]
    c = new_cache(8, 4, 2, H, d, "bf16")
    out = torch.zeros((C, H, d), dtype=torch.bfloat16, device="cuda")
    qd, kd, vd = q.cuda(), k.cuda(), v.cuda()
    for s in range(4):
        c.reserve(s, lens[s])
    # the prompt in one call, then a token of every unfinished segment whose parent is finished
    plan = [([70, 0, 0, 0])] + [[0, int(t < 30), int(t < 20), 0] for t in range(30)] + [[0, 0, 0, 1]] * 25
    at = [0, 0, 0, 0]
    batches = {}
    for new in plan:
        key = tuple(new)
        if key not in batches:
            batches[key] = RolloutBatch(c, parent, new, H)
        b = batches[key]
        rows = torch.tensor([first[s] + at[s] + i for s in range(4) for i in range(new[s])], device="cuda")
        b.advance()
        b.write(kd[rows], vd[rows])
        out[rows] = b.attend(qd[rows])[0]
        at = [a + n for a, n in zip(at, new)]
    assert at == lens
    got = f64(out)
    mag = np.abs(f64(v)).max() * np.ones_like(ref)
    assert np.all(np.abs(got - ref) <= 2.0 ** -8 * (np.abs(ref) + mag) + 2.0 ** -10 * mag)


# ---------------------------------------------------------------------------
# refusals of the Python entry points
# ---------------------------------------------------------------------------

def test_refusals():
    from paper_2608_28158_amd import _lib
    from paper_2608_28158_amd.rollout import RolloutBatch, RolloutCache
    for bad in (dict(kind="int8"), dict(d=96), dict(n_pages=0)):
        a = dict(n_pages=2, n_seg=2, pitch=1, heads=2, d=64, kind="bf16")
        a.update(bad)
        with pytest.raises(ValueError):
            RolloutCache(**a)
    with pytest.raises(RuntimeError):
        RolloutCache(2, 2, 1, 2, 64, device="cpu")
    c = RolloutCache(2, 2, 1, 2, 64)
    x = torch.zeros((1, 2, 64), dtype=torch.bfloat16, device="cuda")
    r = table([(0, 0)])
    for rows, k in ((r, x.float()), (r, x[:, :1]), (r.long(), x), (r, x.cpu()), (r.cpu(), x),
                    (r, torch.zeros((1, 64, 2), dtype=torch.bfloat16, device="cuda").transpose(1, 2))):
        with pytest.raises(ValueError):
            c.write(rows, k, x)
    with pytest.raises(ValueError):
        c.write(r, x, x, layer=1)
    with pytest.raises(RuntimeError):
        c.write(r, x.clone().requires_grad_(), x)
    with torch.no_grad():
        c.write(r, x.clone().requires_grad_(), x)
    with pytest.raises(ValueError):
        RolloutBatch(c, [-1], [1], 2)
    with pytest.raises(_lib.HartsError):
        RolloutBatch(c, [1, 0], [1, 0], 2)
    with pytest.raises(_lib.HartsError):
        RolloutBatch(c, [-1, 0], [1, 0], 3)
    b = RolloutBatch(c, [-1, 0], [1, 0], 4)
    with pytest.raises(ValueError):
        b.attend(x)
    with pytest.raises(ValueError):
        b.attend(torch.zeros((1, 4, 64), dtype=torch.bfloat16, device="cuda"), out=x)
    q = torch.zeros((1, 4, 64), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(_lib.HartsError):
        b.attend(q, out=q)


# ---------------------------------------------------------------------------
# the ends of the types' ranges
# ---------------------------------------------------------------------------

TOP = 2.0 ** 120


@pytest.mark.parametrize("d", [64, 128])
def test_e4m3_of_the_largest_values(d):
    """The nearest code of 248 x 2^120 and more stands for 2^128, which bf16 does not hold: they take
    the largest one that it does, 240 x 2^120."""
    x, want = np.zeros((4, 1, d)), np.zeros((4, 1, d))
    x[0, 0, :6] = [255, -248, 247, 240, -232, 1]            # (232 and 216 lie half way between two codes)
    want[0, 0, :6] = [240, -240, 240, 240, -224, 1]
    x[1, 0, :4] = [-225, 216, 129, np.nan]
    want[1, 0, :4] = [-224, 224, 128, np.nan]
    x[2, 0, :2] = [224, -223]                                # a scale of 2^119: codes of 448 and less
    want[2, 0, :2] = [224, -224]
    x[3] = 255
    want[3] = 240
    b = bf16_values(x * TOP)
    assert np.array_equal(f64(b), x * TOP, equal_nan=True)
    assert np.array_equal(e4m3_vectors(f64(b))[0], want * TOP, equal_nan=True)
    c = new_cache(1, 1, 1, 1, d, "e4m3")
    c.reserve(0, 4)
    c.len[0] = 4
    rows = table([(0, i) for i in range(4)])
    c.write(rows, b.cuda(), b.flip(0).cuda())
    k, v = c.read(rows)
    assert np.array_equal(f64(k), want * TOP, equal_nan=True)
    assert np.array_equal(f64(v)[::-1], want * TOP, equal_nan=True)


@pytest.mark.parametrize("new", [5, 35])
@pytest.mark.parametrize("where", [(0, 10), (1, 41)])
def test_the_largest_values_under_attention(where, new):
    """A value near the type's largest, in a row that all queries see and in a drafted one that some see
    (equal weights: the sum of one such value and ordinary ones is a float32)."""
    from paper_2608_28158_amd.rollout import RolloutBatch
    rng = np.random.default_rng(14)
    d, parent, lens = 64, [-1, 0], [70, 70]
    c, K, V = filled(parent, lens, 2, d, "e4m3", rng)
    k, v = c.read(table([where]))
    v[0, 1, 3:9] = 255 * TOP
    c.write(table([where]), k, v)
    V[where[0]][where[1]] = e4m3_vectors(f64(v))[0][0]
    assert np.isfinite(V[where[0]]).all() and V[where[0]].max() == 240 * TOP
    q = torch.zeros((new, 4, d), dtype=torch.bfloat16)
    o, lse = RolloutBatch(c, parent, [0, new], 4, capacity=lens).attend(q.cuda())
    ref = forest_decode(parent, [0, new], K, V, f64(q), 0.125)
    compare(o, lse, ref, d)


@pytest.mark.parametrize("new", [5, 35])
def test_codes_beyond_bf16(new):
    """Codes that a caller lays into the cache itself and that stand for more than bf16 holds are
    infinities: for the rows that see them, and for no other."""
    from paper_2608_28158_amd.rollout import RolloutBatch
    rng = np.random.default_rng(15)
    d, parent, lens = 64, [-1, 0], [70, 70]
    c, K, V = filled(parent, lens, 2, d, "e4m3", rng)
    at = 70 - new + 3                                        # the fourth of the new rows
    page, slot = int(c.pages[1, at // 64]), at % 64
    c.v.view(torch.uint8)[0, page, 1, slot] = 0x7e           # 448
    c.v_exp[0, page, 1, slot] = 254                          # x 2^127
    assert torch.isinf(c.read(table([(1, at)]))[1][0, 1]).all()
    q = bf16_values(rng.standard_normal((new, 4, d)))
    o, lse = RolloutBatch(c, parent, [0, new], 4, capacity=lens).attend(q.cuda())
    ref = forest_decode(parent, [0, new], K, V, f64(q), 0.125)
    compare(o[:3], lse[:3], [x[:3] for x in ref], d)
    got = f64(o)
    assert np.all(got[3:, 2:] == np.inf)
    assert np.all(np.abs(got[:, :2] - ref[0][:, :2]) <= bounds(ref[0], ref[2], ref[3], ref[1], d)[0][:, :2])


@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,new", [([40], 1), ([2000], 1), ([300, 40], 3), ([300, 90], 40), ([700], 100)])
def test_only_scores_of_minus_infinity(lens, new, d, bad):
    """Rows whose every score is -infinity give zeros, whatever the values of those keys."""
    from paper_2608_28158_amd.rollout import RolloutBatch
    parent = list(range(-1, len(lens) - 1))
    c = new_cache(sum(-(-n // 64) for n in lens), len(lens), -(-max(lens) // 64), 1, d, "bf16")
    for s, n in enumerate(lens):
        c.reserve(s, n)
        c.len[s] = n
        k, v = (torch.zeros((n, 1, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        k[:, 0, 0] = float("-inf")
        v[:] = bad
        c.write(table([(s, p) for p in range(n)]), k, v)
    q = torch.zeros((new, 2, d), dtype=torch.bfloat16, device="cuda")
    q[:, :, 0] = 1
    n_new = [0] * (len(lens) - 1) + [new]
    o, lse = RolloutBatch(c, parent, n_new, 2, capacity=lens).attend(q)
    assert not f64(o).any() and np.all(f64(lse) == -np.inf)


# ---------------------------------------------------------------------------
# autograd, streams, hints
# ---------------------------------------------------------------------------

# ---------------------------------------------------------------------------
# autograd
# ---------------------------------------------------------------------------

def test_writes_are_seen_by_autograd():
    """Tensors that a call writes count as modified: a backward pass that saved one refuses to use it."""
    from paper_2608_28158_amd.rollout import RolloutBatch
    c = new_cache(2, 1, 1, 2, 64, "e4m3")
    c.reserve(0, 3)
    c.len[0] = 3
    x = torch.ones((3, 2, 64), dtype=torch.bfloat16, device="cuda")
    before = [t._version for t in (c.k, c.v, c.k_exp, c.v_exp)]
    c.write(table([(0, i) for i in range(3)]), x, x)
    assert all(t._version > b for t, b in zip((c.k, c.v, c.k_exp, c.v_exp), before))
    w = torch.ones((3, 2, 64), dtype=torch.bfloat16, device="cuda", requires_grad=True)
    out = torch.ones_like(x)
    y = (w * out).sum()
    RolloutBatch(c, [-1], [3], 2).attend(x, out=out)
    with pytest.raises(RuntimeError, match="modified by an inplace"):
        y.backward()


def test_tangents_are_refused():
    import torch.autograd.forward_ad as fwd
    from paper_2608_28158_amd.rollout import RolloutBatch
    c = new_cache(2, 1, 1, 2, 64, "bf16")
    c.reserve(0, 3)
    c.len[0] = 3
    x = torch.ones((3, 2, 64), dtype=torch.bfloat16, device="cuda")
    rows = table([(0, i) for i in range(3)])
    batch = RolloutBatch(c, [-1], [3], 2)
    with fwd.dual_level():
        dual = fwd.make_dual(x, torch.ones_like(x))
        with pytest.raises(RuntimeError, match="not differentiable"):
            c.write(rows, dual, x)
        with pytest.raises(RuntimeError, match="not differentiable"):
            batch.attend(dual)
        c.write(rows, x, x)
        batch.attend(x)


def test_inference_tensors_are_written():
    from paper_2608_28158_amd.rollout import RolloutBatch
    with torch.inference_mode():
        c = new_cache(2, 1, 1, 2, 64, "bf16")
        c.reserve(0, 3)
        c.len[0] = 3
        out = torch.empty((3, 2, 64), dtype=torch.bfloat16, device="cuda")
    x = torch.ones((3, 2, 64), dtype=torch.bfloat16, device="cuda")
    for mode in (torch.inference_mode(), torch.no_grad()):
        with mode:
            c.write(table([(0, i) for i in range(3)]), x, x)
            RolloutBatch(c, [-1], [3], 2).attend(x, out=out)
            assert torch.all(out == 1)


def test_pages_held_are_the_default_capacity():
    from paper_2608_28158_amd.rollout import RolloutBatch
    n = 9
    c = new_cache(400, n, 300, 2, 64, "bf16")
    held = [15000] + [100] * (n - 1)
    for s, rows in enumerate(held):
        c.reserve(s, rows)
    parent, new = [-1] + [0] * (n - 1), [0] + [1] * (n - 1)
    batch = RolloutBatch(c, parent, new, 4)
    same = RolloutBatch(c, parent, new, 4, capacity=[-(-r // 64) * 64 for r in held])
    assert torch.equal(batch._tab, same._tab)
    # a table that the caller fills without reserve(): the most that it can hold
    d = new_cache(4, n, 300, 2, 64, "bf16")
    assert torch.equal(RolloutBatch(d, parent, new, 4)._tab, RolloutBatch(d, parent, new, 4, capacity=[300 * 64] * n)._tab)


def test_tables_outlive_their_batch_on_other_streams():
    """A batch may be dropped while a call on a stream of the caller's is still to run: its tables' memory
    is not handed out before that.  (The new tensors are not written.)"""
    from paper_2608_28158_amd.rollout import RolloutBatch
    rng = np.random.default_rng(18)
    parent, lens, new = FORESTS["long_prefix"]
    c, K, V = filled(parent, lens, 2, 64, "bf16", rng)
    q = bf16_values(rng.standard_normal((9, 4, 64)))
    dev = q.cuda()
    for use in ("attend", "write", "advance"):
        batch = RolloutBatch(c, parent, new, 4, capacity=lens)
        at, n = batch._tab.data_ptr(), batch._tab.numel()
        k = torch.zeros((9, 2, 64), dtype=torch.bfloat16, device="cuda")
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            torch.cuda._sleep(10_000_000)
            if use == "attend":
                o, lse = batch.attend(dev)
            elif use == "write":
                batch.write(k, k)
            else:
                batch.advance()
        del batch
        later = [torch.empty(n, dtype=torch.int32, device="cuda") for _ in range(3)]
        assert at not in [t.data_ptr() for t in later], use
        torch.cuda.synchronize()
        if use == "attend":
            compare(o, lse, forest_decode(parent, new, K, V, f64(q), 0.125), 64)


def test_log_sums_by_graph_replay():
    """The log-sums of captured steps, while the lengths grow."""
    from paper_2608_28158_amd.rollout import RolloutBatch
    rng = np.random.default_rng(16)
    parent, lens, new = [-1, 0, 0], [600, 60, 1], [0, 1, 2]
    c, K, V = filled(parent, lens, 2, 64, "bf16", rng)
    batch = RolloutBatch(c, parent, new, 4, capacity=[600, 80, 80])
    k, v = (torch.zeros((3, 2, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q = torch.zeros((3, 4, 64), dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        batch.advance()
        batch.write(k, v)
        o, lse = batch.attend(q)
    for t in range(4):
        fresh = [bf16_values(rng.standard_normal(tuple(x.shape))) for x in (q, k, v)]
        for x, y in zip((q, k, v), fresh):
            x.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        for j, (s, _) in enumerate(batch.rows.tolist()):
            K[s] = np.concatenate([K[s], f64(fresh[1])[j:j + 1]])
            V[s] = np.concatenate([V[s], f64(fresh[2])[j:j + 1]])
        compare(o, lse, forest_decode(parent, new, K, V, f64(fresh[0]), 0.125), 64)
        eager = batch.attend(q)
        assert torch.equal(eager[0], o) and torch.equal(eager[1], lse)


@pytest.mark.parametrize("d", [64, 128])
def test_the_training_attention_gives_the_same_rows(d):
    """The rows of a finished tree, attended through the cache a segment at a time, against harts_attn_fwd
    over the tree.  Both round the same things (weights to bf16, sums in float32, the output), so they differ
    by at most twice the bound of one."""
    from paper_2608_28158_amd import _lib
    from paper_2608_28158_amd.plan import HartsPlan
    from paper_2608_28158_amd.rollout import RolloutBatch
    from tests.test_gpu_attn import run_attn
    rng = np.random.default_rng(17)
    parent, lens, H = [-1, 0, 0, 1], [150, 70, 20, 65], 2
    n, C = len(lens), sum(lens)
    plan = HartsPlan(parent, lens, 64)
    phys = [np.arange(lens[s]) + int(plan["seg_row"][s]) for s in range(n)]
    q, k, v = (bf16_values(rng.standard_normal((C, H, d))) for _ in range(3))
    trained = run_attn(_lib.lib(), plan, q.cuda(), k.cuda(), v.cuda(), torch.zeros_like(q).cuda(), H, d, d ** -0.5)
    c = new_cache(10, n, 3, H, d, "bf16")
    K, V = [], []
    for s in range(n):                                       # parents come first
        c.reserve(s, lens[s])
        c.len[s] = lens[s]
        new = [lens[s] if i == s else 0 for i in range(n)]
        batch = RolloutBatch(c, parent, new, H, capacity=lens)
        batch.write(k[phys[s]].cuda(), v[phys[s]].cuda())
        K.append(f64(k[phys[s]]))
        V.append(f64(v[phys[s]]))
        o, lse = batch.attend(q[phys[s]].cuda())
        ref = forest_decode(parent[:s + 1], new[:s + 1], K, V, f64(q[phys[s]]), d ** -0.5)
        compare(o, lse, ref, d)
        tol_o, tol_l = bounds(ref[0], ref[2], ref[3], ref[1], d)
        assert np.all(np.abs(f64(o) - f64(trained["o"])[phys[s]]) <= 2 * tol_o)
        assert np.all(np.abs(f64(lse) - f64(trained["lse"])[phys[s]]) <= 2 * tol_l)
