"""Recurrent steps of linear attention and KDA on the GPU, against the float64
oracle.  Tolerances: every sum is float32; of T tokens over d rows each value
passes at most (d + 16) T float32 roundings (16: exponentials, products, the
exchange between lanes), each half a step (2^-24) of a magnitude that the same
sums over absolute values bound; bf16 outputs add their own rounding, 2^-8."""
import numpy as np
import pytest
import torch

from oracle.gen import step_tokens

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")


DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def draw(rng, n, H, d, dtype, kda, states):
    unit = lambda x: x / np.linalg.norm(x, axis=-1, keepdims=True)
    t = lambda x: torch.from_numpy(np.asarray(x, np.float32)).to(DT[dtype])
    x = dict(q=t(unit(rng.standard_normal((n, H, d)))), k=t(unit(rng.standard_normal((n, H, d)))),
             v=t(rng.standard_normal((n, H, d))),
             g=torch.from_numpy(-np.exp(rng.standard_normal((n, H, d) if kda else (n, H)) - 2).astype(np.float32)),
             S=torch.from_numpy(rng.standard_normal((states, H, d, d)).astype(np.float32)))
    if kda:
        x["beta"] = torch.from_numpy(rng.random((n, H)).astype(np.float32))
    return x


def call(kda, x, **kw):
    from paper_2608_28158_amd.rollout import kda_step, la_step
    a = [x[n] if x[n].is_cuda else x[n].cuda() for n in (("q", "k", "v", "g", "beta") if kda else ("q", "k", "v", "g"))]
    return (kda_step if kda else la_step)(*a, **kw)


def num(t):
    return t.detach().cpu().double().numpy()


def check(kda, x, off, src, o, S, dst, scale, dtype):
    """Every sequence's outputs and last state."""
    for i in range(len(off) - 1):
        r = slice(off[i], off[i + 1])
        d = x["q"].shape[2]
        S0 = num(x["S"][src[i]]) if 0 <= src[i] < x["S"].shape[0] else np.zeros((x["q"].shape[1], d, d))
        wo, wS, mo, mS = step_tokens(num(x["q"][r]), num(x["k"][r]), num(x["v"][r]), num(x["g"][r]),
                                     num(x["beta"][r]) if kda else None, S0, scale)
        f = (d + 16) * max(1, off[i + 1] - off[i]) * 2.0 ** -24
        tol = f * mo + (2.0 ** -8 * np.abs(wo) if dtype == "bf16" else 0)
        assert np.all(np.abs(num(o[r]) - wo) <= tol), (i, np.max(np.abs(num(o[r]) - wo) / tol))
        if 0 <= dst[i] < S.shape[0]:
            assert np.all(np.abs(num(S[dst[i]]) - wS) <= f * mS + 1e-30), i


@pytest.mark.parametrize("kda", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H,d", [(1, 64), (3, 128), (5, 64), (16, 128)])
@pytest.mark.parametrize("n", [1, 7])
def test_one_token_in_place(kda, dtype, H, d, n):
    rng = np.random.default_rng(n * d + H)
    x = draw(rng, n, H, d, dtype, kda, n + 2)
    S = x["S"].cuda()
    o = call(kda, x, S=S)
    check(kda, x, range(n + 1), range(n), o, S, range(n), d ** -0.5, dtype)
    assert torch.equal(S[n:].cpu(), x["S"][n:])


@pytest.mark.parametrize("kda", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("tokens", [[3], [0, 1, 0, 5, 2], [33, 1, 7]])
def test_several_tokens_and_a_fork(kda, dtype, d, tokens):
    """Sequences of any number of rows, starting from shared states, into slots of any order."""
    rng = np.random.default_rng(sum(tokens) + d)
    n, H, total = len(tokens), 2, sum(tokens)
    x = draw(rng, total + 3, H, d, dtype, kda, 3)
    off = np.concatenate([[0], np.cumsum(tokens)])
    src = [int(i) for i in rng.integers(0, 3, n)]
    src[-1] = -1 if n > 1 else 2                             # from zeros
    dst = [int(i) for i in rng.permutation(n + 2)[:n]]
    ints = lambda a: torch.tensor(list(a), dtype=torch.int32, device="cuda")
    S_out = torch.full((n + 2, H, d, d), 7.0, device="cuda")
    out = torch.full((total + 3, H, d), 5.0, dtype=DT[dtype], device="cuda")
    S = x["S"].cuda()
    o = call(kda, x, S=S, S_out=S_out, idx_in=ints(src), idx_out=ints(dst), row_off=ints(off), scale=0.7, out=out)
    check(kda, x, off, src, o, S_out, dst, 0.7, dtype)
    assert torch.equal(S.cpu(), x["S"])
    rest = [i for i in range(n + 2) if i not in dst]
    assert torch.all(S_out[rest] == 7) and torch.all(out[total:] == 5)      # what nothing names
    for i, t in enumerate(tokens):
        if t == 0:                                           # handed on, bit for bit
            want = x["S"][src[i]] if src[i] >= 0 else torch.zeros_like(x["S"][0])
            assert torch.equal(S_out[dst[i]].cpu(), want)


@pytest.mark.parametrize("kda", [False, True])
def test_indexes_outside_and_repeated(kda):
    rng = np.random.default_rng(2)
    n, H, d = 70, 2, 64
    x = draw(rng, n, H, d, "f32", kda, n)
    idx = list(range(n))
    idx[3], idx[5], idx[66], idx[69] = -1, 10 ** 9, 2, 2     # no slot, no slot, a repeat of sequence 2, another
    t = torch.tensor(idx, dtype=torch.int32, device="cuda")
    S = x["S"].cuda()
    o = call(kda, x, S=S, idx_in=t)
    good = [i for i in range(n) if i not in (66, 69)]
    y = {m: (v[good] if m != "S" else v) for m, v in x.items()}
    check(kda, y, range(len(good) + 1), [idx[i] for i in good], o[good], S, [idx[i] for i in good], d ** -0.5, "f32")
    assert torch.isnan(o[[66, 69]]).all()
    keep = [i for i in range(n) if i not in idx]
    assert torch.equal(S[keep].cpu(), x["S"][keep])
    # into another pool, a repeat writes nothing either
    S_out = torch.full((4, H, d, d), 3.0, device="cuda")
    o2 = call(kda, {m: (v[:4] if m != "S" else v) for m, v in x.items()}, S=x["S"].cuda(), S_out=S_out,
              idx_out=torch.tensor([1, 0, 1, 4], dtype=torch.int32, device="cuda"))
    assert torch.isnan(o2[2]).all() and torch.isfinite(o2[[0, 1, 3]]).all() and torch.all(S_out[2:] == 3)


@pytest.mark.parametrize("kda", [False, True])
def test_pools_past_32_bits(kda):
    """States past 2^31 elements, and the variant that goes around the cache (more than 128 MiB of states)."""
    rng = np.random.default_rng(6)
    H, d, n, slots = 16, 128, 160, 8300
    assert (slots - n) * H * d * d > 2 ** 31 - 2 ** 26 and n * H * d * d * 4 > 128 << 20
    x = draw(rng, n, H, d, "bf16", kda, 1)
    S = torch.zeros((slots, H, d, d), device="cuda")
    first = torch.from_numpy(rng.standard_normal((2, H, d, d)).astype(np.float32)).cuda()
    idx = torch.arange(slots - n, slots, dtype=torch.int32, device="cuda").flip(0).contiguous()
    S[slots - 1], S[slots - n] = first[0], first[1]
    o = call(kda, x, S=S, idx_in=idx)
    for i, s0 in ((0, first[0]), (n - 1, first[1]), (n // 2, torch.zeros_like(first[0]))):
        y = {m: (v[i:i + 1] if m != "S" else s0.cpu()[None]) for m, v in x.items()}
        check(kda, y, [0, 1], [0], o[i:i + 1], S[int(idx[i])][None], [0], d ** -0.5, "bf16")


@pytest.mark.parametrize("kda", [False, True])
def test_decays_of_zero_and_minus_infinity(kda):
    rng = np.random.default_rng(4)
    x = draw(rng, 2, 1, 64, "f32", kda, 2)
    x["g"][0] = 0
    x["g"][1] = -float("inf")
    S = x["S"].cuda()
    o = call(kda, x, S=S)
    check(kda, x, range(3), range(2), o, S, range(2), 0.125, "f32")


@pytest.mark.parametrize("kda", [False, True])
def test_no_sequences(kda):
    x = draw(np.random.default_rng(0), 0, 2, 64, "f32", kda, 1)
    S = x["S"].cuda()
    assert call(kda, x, S=S).shape == (0, 2, 64) and torch.equal(S.cpu(), x["S"])
    zero = torch.zeros(1, dtype=torch.int32, device="cuda")
    assert call(kda, x, S=S, row_off=zero).shape == (0, 2, 64)


@pytest.mark.parametrize("kda", [False, True])
def test_steps_by_graph_replay(kda):
    rng = np.random.default_rng(9)
    n, H, d = 5, 2, 64
    x = draw(rng, n, H, d, "bf16", kda, n)
    dev = {m: t.cuda() for m, t in x.items()}
    S, E = dev.pop("S"), x["S"].cuda()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        o = call(kda, dev, S=S)
    for t in range(4):
        y = draw(rng, n, H, d, "bf16", kda, n)
        for m in dev:
            dev[m].copy_(y[m])
        graph.replay()
        want = call(kda, dev, S=E)
        torch.cuda.synchronize()
        assert torch.equal(o, want) and torch.equal(S, E)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_prompt_by_chunks_then_tokens_la(dtype):
    """A prompt through the chunked training form, its rollouts token by token from the prompt's final
    state, against the training form over the whole tree (both within rounding of the exact recurrence)."""
    from paper_2608_28158_amd.plan import HartsPlan
    from paper_2608_28158_amd.tree_la import tree_la
    rng = np.random.default_rng(21)
    H, d, lens = 2, 64, [100, 9, 9, 9]
    x = draw(rng, sum(lens), H, d, dtype, False, 1)
    q, k, v, g = (x[m].cuda() for m in ("q", "k", "v", "g"))
    whole = HartsPlan([-1, 0, 0, 0], lens)
    rows = [torch.arange(int(whole["seg_row"][s]), int(whole["seg_row"][s]) + lens[s], device="cuda") for s in range(4)]
    o_all, _ = tree_la(q, k, v, g, whole)
    prompt = HartsPlan([-1], [100])
    p = rows[0]
    _, S0 = tree_la(q[p], k[p], v[p], g[p], prompt)
    S = torch.empty((3, H, d, d), device="cuda")
    tok = torch.stack(rows[1:])                              # [3, 9]
    for t in range(9):
        r = tok[:, t]
        y = dict(q=q[r], k=k[r], v=v[r], g=g[r])
        if t == 0:                                           # the fork
            o = call(False, y, S=S0, S_out=S, idx_in=torch.zeros(3, dtype=torch.int32, device="cuda"))
        else:
            o = call(False, y, S=S)
        a, b = num(o), num(o_all[r])
        tol = 1e-4 if dtype == "f32" else 2e-2               # the training form's own tolerance
        assert np.max(np.abs(a - b)) <= tol * np.max(np.abs(num(o_all))), t


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_prompt_by_chunks_then_tokens_kda(dtype):
    from paper_2608_28158_amd.kda import KdaRunner
    from paper_2608_28158_amd.plan import HartsPlan
    rng = np.random.default_rng(22)
    H, d, lens = 2, 64, [100, 9, 9]
    x = draw(rng, sum(lens), H, d, dtype, True, 1)
    dev = {m: x[m].cuda() for m in ("q", "k", "v", "g", "beta")}
    zero = torch.zeros((1, H, d, d), device="cuda")
    whole = HartsPlan([-1, 0, 0], lens)
    o_all, _ = KdaRunner(whole, H, d, DT[dtype]).forward(*dev.values(), zero, d ** -0.5)
    rows = [torch.arange(int(whole["seg_row"][s]), int(whole["seg_row"][s]) + lens[s], device="cuda") for s in range(3)]
    _, S0 = KdaRunner(HartsPlan([-1], [100]), H, d, DT[dtype]).forward(*(t[rows[0]] for t in dev.values()), zero,
                                                                       d ** -0.5)
    # all of a rollout's tokens in one call, from the prompt's state
    r = torch.cat(rows[1:])
    S = torch.empty((2, H, d, d), device="cuda")
    ints = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
    o = call(True, {m: t[r] for m, t in dev.items()}, S=S0, S_out=S, idx_in=ints([0, 0]), row_off=ints([0, 9, 18]))
    tol = 1e-4 if dtype == "f32" else 2e-2
    assert np.max(np.abs(num(o) - num(o_all[r]))) <= tol * np.max(np.abs(num(o_all)))


def test_refusals():
    from paper_2608_28158_amd import _lib
    x = draw(np.random.default_rng(0), 2, 2, 64, "bf16", False, 2)
    S = x["S"].cuda()
    ints = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
    for over in (dict(q=x["q"].half()), dict(k=x["k"].float()), dict(g=x["g"].double()), dict(v=x["v"][:1]),
                 dict(g=x["g"].cpu().t().contiguous().t())):
        with pytest.raises(ValueError):
            call(False, {**x, **over}, S=S)
    for kw in (dict(S=S[:1]), dict(S=S, idx_out=ints([0, 1])), dict(S=S, idx_in=ints([0])),
               dict(S=S, idx_in=ints([0, 1]).long()), dict(S=S.double()), dict(S=S, row_off=ints([])),
               dict(S=S, row_off=torch.tensor([0, 2], dtype=torch.int32))):
        with pytest.raises(ValueError):
            call(False, x, **kw)
    with pytest.raises(ValueError, match="beta"):
        call(True, {**x, "g": x["q"].float(), "beta": S.new_empty(0)}, S=S)
    from paper_2608_28158_amd.rollout import kda_step
    with pytest.raises(ValueError, match="beta"):
        kda_step(*(x[n].cuda() for n in "qkv"), x["q"].float().cuda(), None, S)
    with pytest.raises(RuntimeError):
        call(False, {**x, "v": x["v"].cuda().requires_grad_()}, S=S)
    with pytest.raises(ValueError):
        call(False, x, S=S, S_out=S, idx_out=ints([1, 0]))
    with pytest.raises(_lib.HartsError):
        call(False, x, S=S, S_out=S.view(2, 2, 64, 64), idx_out=ints([1, 0]))
    v = x["v"].cuda()
    with pytest.raises(_lib.HartsError):
        call(False, {**x, "v": v}, S=S, out=v)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gates_of_any_float_alignment(dtype):
    """A token's slice of gates [tokens, H], H no multiple of 4 (linear attention reads them one by one)."""
    rng = np.random.default_rng(31)
    H, d = 5, 64
    x = draw(rng, 3, H, d, dtype, False, 1)
    g = x["g"].cuda()
    for t in range(3):
        y = {m: (v[t:t + 1] if m != "S" else v) for m, v in x.items()}
        y["q"], y["k"], y["v"] = (y[m].clone() for m in "qkv")
        S = x["S"].cuda()
        assert t == 0 or g[t:t + 1].data_ptr() % 16 != 0
        o = call(False, {**y, "g": g[t:t + 1]}, S=S)
        check(False, y, [0, 1], [0], o, S, [0], d ** -0.5, dtype)


@pytest.mark.parametrize("kda", [False, True])
def test_writes_are_seen_by_autograd(kda):
    x = draw(np.random.default_rng(32), 2, 2, 64, "f32", kda, 2)
    w = torch.ones((2, 2, 64), device="cuda", requires_grad=True)
    out, S, S_out = torch.ones((2, 2, 64), device="cuda"), x["S"].cuda(), x["S"].cuda()
    y = (w * out).sum()
    call(kda, x, S=S, out=out)
    with pytest.raises(RuntimeError, match="modified by an inplace"):
        y.backward()
    a, b = S._version, S_out._version
    call(kda, x, S=S, S_out=S_out)
    assert S._version == a and S_out._version > b            # (only read, written)
    call(kda, x, S=S)
    assert S._version > a
    with torch.inference_mode():
        S = x["S"].cuda()
    call(kda, x, S=S)                                        # (has no version)


@pytest.mark.parametrize("kda", [False, True])
def test_tangents_are_refused(kda):
    import torch.autograd.forward_ad as fwd
    x = draw(np.random.default_rng(33), 2, 2, 64, "f32", kda, 2)
    S = x["S"].cuda()
    with fwd.dual_level():
        v = x["v"].cuda()
        with pytest.raises(RuntimeError, match="not differentiable"):
            call(kda, {**x, "v": fwd.make_dual(v, torch.ones_like(v))}, S=S)
        with pytest.raises(RuntimeError, match="not differentiable"):
            call(kda, x, S=fwd.make_dual(S, torch.ones_like(S)))
        call(kda, x, S=S)
