"""Measured cases of the generation operators: a paged key/value cache that is
quantised as it is written and read back, attention of new rows over a forest
of cached segments (a shared prefix computed once for all rows below it), and
the recurrent steps of linear attention and of KDA.

A case is a dict of plain values.  ``prepare`` draws its inputs on the GPU,
``run`` is one pass: the operators' plain form in elementary torch, or, where
``own`` is true, the calls of a program that generates with the library.
``exact`` is the same pass in float64.

Forests: ``prompts`` roots of about ``prefix`` rows; below each, ``branches``
inner segments (none if 0), below each of those (or the root) ``samples``
leaves of up to ``tail`` rows.  The last 1 to ``new`` rows of every leaf are
the pass's queries.  With no samples the roots are the leaves.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

PAGE = 64                                  # rows of a cache page
E4M3_MAX = 448.0


def _attn(name, kind, q_heads, kv_heads, d, prompts, prefix, branches, samples, tail, new, fseed):
    return dict(name=name, op="attn", kind=kind, q_heads=q_heads, kv_heads=kv_heads, d=d, prompts=prompts,
                prefix=prefix, branches=branches, samples=samples, tail=tail, new=new, fseed=fseed)


def _cache(name, kind, heads, d, seqs, most, fseed):
    return dict(name=name, op="cache", kind=kind, heads=heads, d=d, seqs=seqs, most=most, fseed=fseed)


def _step(name, op, dtype, heads, d, seqs, siblings, tokens, fseed):
    return dict(name=name, op=op, dtype=dtype, heads=heads, d=d, seqs=seqs, siblings=siblings, tokens=tokens,
                fseed=fseed)


def listed():
    return [
        # one token of one sequence enters an 8-bit cache and is read back: latency
        _cache("cache_one_e4m3", "e4m3", 16, 128, 1, 1, 0),
        # one token of each of 192 rollouts in flight, small heads
        _cache("cache_192_tokens", "e4m3", 20, 64, 192, 1, 1),
        # the prompts of a microbatch enter the cache and are read back for a training kernel
        _cache("cache_prompts_30k", "e4m3", 16, 128, 12, 4999, 2),
        # the first tokens of one rollout: latency of a lone short sequence
        _attn("attn_one_short", "bf16", 16, 16, 128, 1, 333, 0, 0, 0, 1, 0),
        # one generated token of 4 prompts with 16 rollouts each, every head with keys of its own
        _attn("attn_4x16_8k", "bf16", 16, 16, 128, 4, 8192, 0, 16, 1500, 1, 1),
        # one generated token of 64 rollouts of one long agentic context, 8-bit cache, 4 query heads a key head
        _attn("attn_1x64_64k_e4m3", "e4m3", 32, 8, 128, 1, 65000, 0, 64, 3900, 1, 2),
        # several drafted tokens at the ends of branching rollouts, small heads
        _attn("attn_branches_drafts", "bf16", 20, 5, 64, 6, 2500, 3, 4, 700, 9, 3),
        # the next 2,000 rows or fewer of long prompts against what the cache holds
        _attn("attn_prompt_chunk", "bf16", 16, 4, 128, 3, 14000, 0, 0, 0, 2000, 4),
        # one token of one sequence in float32: latency
        _step("la_step_one_f32", "la", "f32", 4, 64, 1, 1, 1, 0),
        # one token of each of 512 rollouts
        _step("la_step_512", "la", "bf16", 16, 128, 512, 1, 1, 1),
        # the first tokens of 8 samples of each of 3 prompts, all starting from their prompt's state
        _step("kda_step_fork_f32", "kda", "f32", 8, 64, 24, 8, 5, 2),
        # one token of each of 256 rollouts
        _step("kda_step_256", "kda", "bf16", 16, 128, 256, 1, 1, 3),
    ]


def draw(rng):
    """One more case of the ranges of the listed ones, of no more work than the largest of them."""
    while True:
        c = _draw(rng)
        w = work(c)
        if w["bytes"] <= 1.0e9 and w["flops"] <= 3.5e11:
            return c


def _draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["cache", "attn", "attn", "attn", "la", "kda"])
    fseed = rng.randrange(1 << 30)
    d = rng.choice([64, 128, 128])
    if op == "cache":
        seqs = log(1, 256)
        c = _cache("", rng.choice(["e4m3", "e4m3", "bf16"]), rng.choice([1, 2, 4, 5, 8, 12, 16, 20]), d, seqs,
                   1 if rng.random() < 0.4 else log(1, max(1, 50000 // seqs)), fseed)
    elif op == "attn":
        kv = rng.choice([1, 2, 4, 5, 8, 8, 16])
        group = rng.choice([1, 1, 2, 3, 4, 8])
        group = min(group, 32 // kv)
        kind = rng.choice(["bf16", "e4m3"])
        shape = rng.choice(["one", "samples", "samples", "branches", "chunk"])
        prompts = log(1, 8)
        if shape == "one":
            c = _attn("", kind, kv * group, kv, d, log(1, 48), log(1, 20000), 0, 0, 0, rng.choice([1, 1, 4]), fseed)
        elif shape == "chunk":
            c = _attn("", kind, kv * group, kv, d, min(prompts, 3), log(30, 10000), 0, 0, 0, log(16, 2000), fseed)
        else:
            c = _attn("", kind, kv * group, kv, d, prompts, log(100, 64000 // prompts),
                      0 if shape == "samples" else rng.randint(2, 4), rng.randint(2, 64 // prompts + 1), log(1, 3000),
                      rng.choice([1, 1, 1, 2, 9]), fseed)
            if shape == "branches":
                c["samples"] = min(c["samples"], 6)
    else:
        seqs = log(1, 512 if op == "la" else 256)
        siblings = rng.choice([1, 1, min(seqs, 4), min(seqs, 16)])
        c = _step("", op, rng.choice(["bf16", "bf16", "f32"]), rng.choice([1, 2, 4, 5, 8, 16, 16]), d, seqs, siblings,
                  rng.choice([1, 1, 1, 3, 8]), fseed)
    del c["name"]
    return c


# ---------------------------------------------------------------------------
# structure of a case (from the case alone)
# ---------------------------------------------------------------------------

def _forest(case):
    """(parent, rows, new) of every segment; parents come before their children."""
    r = random.Random(case["fseed"])
    parent, rows, new = [], [], []

    def add(p, n, m):
        parent.append(p)
        rows.append(n)
        new.append(m)
        return len(rows) - 1

    def leaf_new(n):
        # (a single row is the generated token; more are drafts, or the rows of a prompt)
        return min(n, r.randint(max(1, case["new"] // 2), case["new"]))

    for _ in range(case["prompts"]):
        n = case["prefix"] if case["prompts"] == 1 else max(1, int(case["prefix"] * r.uniform(0.6, 1.4)))
        if not case["samples"]:
            add(-1, n, leaf_new(n))
            continue
        root = add(-1, n, 0)
        heads = [add(root, r.randint(1, case["tail"]), 0) for _ in range(case["branches"])] or [root]
        for h in heads:
            for _ in range(case["samples"]):
                n = r.randint(1, case["tail"])
                add(h, n, leaf_new(n))
    return parent, rows, new


def _chain(parent, s):
    """Ancestors of s from the root, s last."""
    out = [s]
    while parent[out[-1]] >= 0:
        out.append(parent[out[-1]])
    return out[::-1]


def _lengths(case):
    """Rows that each sequence holds already and rows that it adds (cache cases), or tokens of each (steps)."""
    r = random.Random(case["fseed"])
    if case["op"] == "cache":
        add = [case["most"] if case["seqs"] == 1 or case["most"] == 1 else r.randint(1, case["most"])
               for _ in range(case["seqs"])]
        return [r.randint(0, 700) for _ in add], add
    return [case["tokens"] if case["tokens"] == 1 else r.randint(1, case["tokens"]) for _ in range(case["seqs"])]


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _quantise(x):
    """e4m3 codes (as float8 values) and biased scale exponents of vectors x
    [..., d] (float32): the scale is the smallest power of two, at least
    2^-126, that brings the largest magnitude to 448 or less."""
    top = x.abs().amax(-1)
    m, e = torch.frexp(top)                                   # top = m 2^e, m in [0.5, 1); 448 = 0.875 2^9
    e = torch.where(m <= 0.875, e - 9, e - 8)
    e = torch.where(top == 0, torch.full_like(e, -126), e.clamp(min=-126))
    inv = ((127 - e) << 23).view(torch.float32)               # 2^-e
    return (x * inv[..., None]).to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def _scale(b):
    """2^(b - 127) of biased exponents b >= 1."""
    return (b.to(torch.int32) << 23).view(torch.float32)


def _make_cache(case, rows, heads, gen):
    """Pages in random order with old rows in all of them, the table and lengths."""
    d, dev = case["d"], "cuda"
    need = [-(-n // PAGE) for n in rows]
    n_pages, pitch = sum(need) + 3, max(need)
    order = torch.randperm(n_pages, generator=gen, device=dev).to(torch.int32)
    table = torch.full((len(rows), pitch), -1, dtype=torch.int32, device=dev)
    at = np.concatenate([[0], np.cumsum(need)])
    for s, n in enumerate(need):
        table[s, :n] = order[int(at[s]):int(at[s + 1])]
    st = dict(n_pages=n_pages, pitch=pitch, table=table,
              len=torch.tensor(rows, dtype=torch.int32, device=dev), k_exp=None, v_exp=None)
    for name in ("k", "v"):
        x = torch.empty((n_pages, heads, PAGE, d), dtype=torch.bfloat16, device=dev)
        for p0 in range(0, n_pages, 256):                     # (in pieces: the float32 draw is twice the cache)
            p1 = min(n_pages, p0 + 256)
            y = torch.randn((p1 - p0, heads, PAGE, d), generator=gen, device=dev)
            if name == "k":                                   # a few channels of keys are larger than the others
                y[..., ::29] *= 4.0
            x[p0:p1] = y
        if case["kind"] == "e4m3":
            c = torch.empty(x.shape, dtype=torch.float8_e4m3fn, device=dev)
            b = torch.empty(x.shape[:-1], dtype=torch.uint8, device=dev)
            for p0 in range(0, n_pages, 256):
                p1 = min(n_pages, p0 + 256)
                c[p0:p1], b[p0:p1] = _quantise(x[p0:p1].float())
            st[name], st[name + "_exp"] = c, b
        else:
            st[name] = x
    return st


def _own_cache(st, case, heads):
    from paper_2608_28158_amd.rollout import RolloutCache
    cache = RolloutCache(st["n_pages"], st["table"].shape[0], st["pitch"], heads, case["d"], kind=case["kind"])
    cache.k[0].copy_(st["k"])
    cache.v[0].copy_(st["v"])
    if case["kind"] == "e4m3":
        cache.k_exp[0].copy_(st["k_exp"])
        cache.v_exp[0].copy_(st["v_exp"])
    cache.pages.copy_(st["table"])
    cache.len.copy_(st["len"])
    return cache


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    d = case["d"]

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    if case["op"] == "cache":
        held, add = _lengths(case)
        heads = case["heads"]
        st = _make_cache(case, [a + b for a, b in zip(held, add)], heads, gen)
        # rows (sequence, position counted from the sequence's end), the new ones of each in order
        rows = [(s, j - n) for s, n in enumerate(add) for j in range(n)]
        st["rows"] = torch.tensor(rows, dtype=torch.int32, device="cuda").reshape(-1, 2)
        st["k_new"], st["v_new"] = (normal(len(rows), heads, d).to(torch.bfloat16) for _ in range(2))
        if own:
            cache = _own_cache(st, case, heads)
            st = dict(cache=cache, rows=st["rows"], k_new=st["k_new"], v_new=st["v_new"])
        return dict(st, case=case)
    if case["op"] == "attn":
        parent, rows, new = _forest(case)
        st = _make_cache(case, rows, case["kv_heads"], gen)
        st["q"] = normal(sum(new), case["q_heads"], d).to(torch.bfloat16)
        if own:
            from paper_2608_28158_amd.rollout import RolloutBatch
            cache = _own_cache(st, case, case["kv_heads"])
            batch = RolloutBatch(cache, parent, new, case["q_heads"], capacity=rows)
            st = dict(cache=cache, batch=batch, q=st["q"])
        else:
            st["forest"] = (parent, rows, new)
        return dict(st, case=case)

    # steps: states of the prompts in one pool, those after the pass in another, in slots of any order
    tokens, heads, n = _lengths(case), case["heads"], case["seqs"]
    dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    n_in = -(-n // case["siblings"])
    total = sum(tokens)
    unit = torch.nn.functional.normalize
    st = dict(q=unit(normal(total, heads, d), dim=-1).to(dt), k=unit(normal(total, heads, d), dim=-1).to(dt),
              v=normal(total, heads, d).to(dt), S_in=normal(n_in, heads, d, d),
              S_out=torch.zeros((n, heads, d, d), device="cuda"))
    src = torch.randperm(n_in, generator=gen, device="cuda")
    st["idx_in"] = src.repeat_interleave(case["siblings"])[:n].to(torch.int32)
    st["idx_out"] = torch.randperm(n, generator=gen, device="cuda").to(torch.int32)
    off = np.concatenate([[0], np.cumsum(tokens)])
    st["row_off"] = torch.tensor(off, dtype=torch.int32, device="cuda") if case["tokens"] > 1 else None
    if case["op"] == "la":
        # decays of about 0.9 to 0.999 a token
        st["g"] = -torch.exp(normal(total, heads) - 4.0)
    else:
        st["g"] = -torch.exp(normal(total, heads, d) - 4.0)
        st["beta"] = torch.sigmoid(normal(total, heads))
    return dict(st, case=case, tokens=tokens)


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(state):
    case = state["case"]
    if own:
        return _run_own(state, case)
    if case["op"] == "cache":
        return _plain_cache(state, case)
    if case["op"] == "attn":
        return _plain_attn(state, case)
    return _plain_step(state, case)


def _run_own(st, case):
    from paper_2608_28158_amd.rollout import kda_step, la_step
    if case["op"] == "cache":
        st["cache"].write(st["rows"], st["k_new"], st["v_new"])
        return st["cache"].read(st["rows"])
    if case["op"] == "attn":
        return st["batch"].attend(st["q"])
    if case["op"] == "la":
        o = la_step(st["q"], st["k"], st["v"], st["g"], st["S_in"], S_out=st["S_out"], idx_in=st["idx_in"],
                    idx_out=st["idx_out"], row_off=st["row_off"])
    else:
        o = kda_step(st["q"], st["k"], st["v"], st["g"], st["beta"], st["S_in"], S_out=st["S_out"],
                     idx_in=st["idx_in"], idx_out=st["idx_out"], row_off=st["row_off"])
    return o, st["S_out"]


def _plain_cache(st, case):
    seg, pos = st["rows"].long().unbind(1)
    pos = torch.where(pos < 0, pos + st["len"][seg].long(), pos)
    page = st["table"][seg, pos // PAGE].long()
    slot = pos % PAGE
    out = []
    for name in ("k", "v"):
        if case["kind"] == "e4m3":
            code, b = _quantise(st[name + "_new"].float())
            st[name].view(torch.uint8)[page, :, slot] = code.view(torch.uint8)
            st[name + "_exp"][page, :, slot] = b
            back = st[name].view(torch.uint8)[page, :, slot].view(torch.float8_e4m3fn).float()
            out.append((back * _scale(st[name + "_exp"][page, :, slot])[..., None]).to(torch.bfloat16))
        else:
            st[name][page, :, slot] = st[name + "_new"]
            out.append(st[name][page, :, slot])
    return tuple(out)


def _chain_rows(st, name, segs, rows, dtype):
    """[heads, keys, d] of the segments' cached rows, one after the other."""
    parts = []
    for s in segs:
        pages = st["table"][s, :-(-rows[s] // PAGE)].long()
        if st[name + "_exp"] is not None:
            x = st[name].view(torch.uint8)[pages].view(torch.float8_e4m3fn).to(dtype)
            x = x * _scale(st[name + "_exp"][pages]).to(dtype)[..., None]
        else:
            x = st[name][pages].to(dtype)
        parts.append(x.transpose(0, 1).reshape(x.shape[1], -1, x.shape[3])[:, :rows[s]])
    return torch.cat(parts, 1)


def _plain_attn(st, case):
    """Each sequence on its own: its whole chain of keys, a masked softmax, the weighted values."""
    parent, rows, new = st["forest"]
    q, Hk, d = st["q"], case["kv_heads"], case["d"]
    group = case["q_heads"] // Hk
    o = torch.empty_like(q)
    lse = torch.empty(q.shape[:2], dtype=torch.float32, device=q.device)
    r0 = 0
    for s, n in enumerate(new):
        if n == 0:
            continue
        segs = _chain(parent, s)
        K = _chain_rows(st, "k", segs, rows, torch.float32)
        V = _chain_rows(st, "v", segs, rows, torch.float32)
        N = K.shape[1]
        x = q[r0:r0 + n].float().reshape(n, Hk, group, d).permute(1, 0, 2, 3).reshape(Hk, n * group, d)
        z = torch.matmul(x, K.transpose(1, 2).contiguous()).reshape(Hk, n, group, N) * d ** -0.5
        if n > 1:
            seen = torch.arange(N, device=q.device)[None] <= torch.arange(N - n, N, device=q.device)[:, None]
            z = z.masked_fill(~seen[None, :, None], float("-inf"))
        top = z.amax(-1, keepdim=True)
        w = torch.exp(z - top)
        total = w.sum(-1, keepdim=True)
        y = torch.matmul((w / total).reshape(Hk, n * group, N), V).reshape(Hk, n, group, d)
        o[r0:r0 + n] = y.permute(1, 0, 2, 3).reshape(n, Hk * group, d).to(o.dtype)
        lse[r0:r0 + n] = (top + torch.log(total))[..., 0].permute(1, 0, 2).reshape(n, Hk * group)
        r0 += n
    return o, lse


def _plain_step(st, case):
    """Token by token over the sequences that have one left."""
    tokens, d = st["tokens"], case["d"]
    q, k, v, g = (st[n].float() for n in ("q", "k", "v", "g"))
    S = st["S_in"][st["idx_in"].long()]
    o = torch.empty_like(q)
    off = np.concatenate([[0], np.cumsum(tokens)])[:-1]
    most = max(tokens)
    for t in range(most):
        if most == 1:
            live, rows, X = slice(None), slice(None), S
        else:
            seqs = [i for i, n in enumerate(tokens) if n > t]
            live = torch.tensor(seqs, device=q.device)
            rows = torch.tensor([int(off[i]) + t for i in seqs], device=q.device)
            X = S[live]
        kt, vt, a = k[rows], v[rows], torch.exp(g[rows])
        if case["op"] == "la":
            X = a[..., None, None] * X + kt[..., :, None] * vt[..., None, :]
        else:
            X = a[..., :, None] * X
            delta = st["beta"][rows][..., None] * (vt - (kt[..., :, None] * X).sum(-2))
            X = X + kt[..., :, None] * delta[..., None, :]
        o[rows] = (q[rows][..., :, None] * X).sum(-2) * d ** -0.5
        if most == 1:
            S = X
        else:
            S[live] = X
    st["S_out"][st["idx_out"].long()] = S
    return o.to(st["q"].dtype), st["S_out"]


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    if case["op"] == "cache":
        n = sum(_lengths(case)[1]) * case["heads"]
        held = n * (case["d"] + 1 if case["kind"] == "e4m3" else 2 * case["d"])
        # k and v: read, written to the cache, read from it, written out
        return {"bytes": 2 * (2 * held + 2 * n * case["d"] * 2) + 8 * (n // case["heads"]), "flops": 0}
    if case["op"] == "attn":
        parent, rows, new = _forest(case)
        used, pairs = set(), 0
        for s, n in enumerate(new):
            if n:
                segs = _chain(parent, s)
                used.update(segs)
                N = sum(rows[c] for c in segs)
                pairs += n * N - n * (n - 1) // 2
        d, held = case["d"], 2 * case["d"] if case["kind"] == "bf16" else case["d"] + 1
        return {"bytes": 2 * case["kv_heads"] * held * sum(rows[s] for s in used)
                + sum(new) * case["q_heads"] * (4 * d + 4),
                "flops": 4 * d * case["q_heads"] * pairs}
    H, d, n = case["heads"], case["d"], case["seqs"]
    total, el = sum(_lengths(case)), 4 if case["dtype"] == "f32" else 2
    states = (n + -(-n // case["siblings"])) * H * d * d * 4
    rows = total * H * (4 * d * el + (4 if case["op"] == "la" else 4 * d + 4))
    return {"bytes": states + rows, "flops": total * H * d * d * (5 if case["op"] == "la" else 7)}


# ---------------------------------------------------------------------------
# the definition in float64
# ---------------------------------------------------------------------------

def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    if case["op"] == "cache":
        return tuple(_exact_held(st[n], case["kind"]) for n in ("k_new", "v_new"))
    return _exact_attn(st, case) if case["op"] == "attn" else _exact_step(st, case)


def _exact_held(x, kind):
    """The value that the cache stands for: x rounded to 4 significant bits
    (steps no finer than 2^-9 of the scale), to nearest, ties to even."""
    x = x.double()
    if kind == "bf16":
        return x
    out = torch.empty_like(x)
    for r0 in range(0, x.shape[0], 4096):
        y = x[r0:r0 + 4096]
        top = y.abs().amax(-1, keepdim=True)
        e = torch.ceil(torch.log2(top.clamp(min=1e-300) / E4M3_MAX))
        e = torch.where(torch.exp2(e - 1) * E4M3_MAX >= top, e - 1, e)     # (log2 next to a power of two)
        e = torch.where(torch.exp2(e) * E4M3_MAX < top, e + 1, e).clamp(min=-126)
        z = y * torch.exp2(-e)
        low = torch.floor(torch.log2(z.abs().clamp(min=2.0 ** -6)))
        low = torch.where(torch.exp2(low) > z.abs().clamp(min=2.0 ** -6), low - 1, low)
        low = torch.where(torch.exp2(low + 1) <= z.abs(), low + 1, low)
        step = torch.exp2(low - 3)
        out[r0:r0 + 4096] = torch.round(z / step) * step * torch.exp2(e)
    return out


def _exact_attn(st, case):
    parent, rows, new = st["forest"]
    Hq, Hk, d = case["q_heads"], case["kv_heads"], case["d"]
    q = st["q"].double()
    o, lse = torch.empty_like(q), torch.empty(q.shape[:2], dtype=torch.float64, device=q.device)
    r0 = 0
    for s, n in enumerate(new):
        if not n:
            continue
        segs = _chain(parent, s)
        N = sum(rows[c] for c in segs)
        where = torch.cat([torch.stack([torch.full((rows[c],), c, device=q.device),
                                        torch.arange(rows[c], device=q.device)], 1) for c in segs])
        page = st["table"][where[:, 0], torch.div(where[:, 1], PAGE, rounding_mode="floor")].long()
        slot = where[:, 1] % PAGE
        for h in range(Hk):
            kv = []
            for name in ("k", "v"):
                if case["kind"] == "e4m3":
                    x = st[name].view(torch.uint8)[page, h, slot].view(torch.float8_e4m3fn).double()
                    x = x * torch.exp2(st[name + "_exp"][page, h, slot].double() - 127.0)[:, None]
                else:
                    x = st[name][page, h, slot].double()
                kv.append(x)
            for p0 in range(0, n, 256):
                p1 = min(n, p0 + 256)
                last = torch.arange(N - n + p0, N - n + p1, device=q.device)
                hide = torch.arange(N, device=q.device)[None] > last[:, None]
                for j in range(h * Hq // Hk, (h + 1) * Hq // Hk):
                    z = (q[r0 + p0:r0 + p1, j] @ kv[0].t()) / math.sqrt(d)
                    z[hide] = -math.inf
                    lse[r0 + p0:r0 + p1, j] = torch.logsumexp(z, 1)
                    o[r0 + p0:r0 + p1, j] = torch.softmax(z, 1) @ kv[1]
        r0 += n
    return o, lse


def _exact_step(st, case):
    n, H, d = case["seqs"], case["heads"], case["d"]
    q, k, v, g = (st[x].double() for x in ("q", "k", "v", "g"))
    o = torch.empty_like(q)
    out = torch.empty(st["S_out"].shape, dtype=torch.float64, device=q.device)
    first = np.concatenate([[0], np.cumsum(st["tokens"])])
    for h in range(H):
        S = st["S_in"][st["idx_in"].long(), h].double()
        for t in range(max(st["tokens"])):
            at = np.array([i for i in range(n) if st["tokens"][i] > t])
            r = torch.from_numpy(first[at] + t).to(q.device)
            at = torch.from_numpy(at).to(q.device)
            X = torch.exp(g[r, h]).reshape(len(r), -1, 1) * S[at]
            new = v[r, h]
            if case["op"] == "kda":
                new = st["beta"][r, h].double()[:, None] * (new - torch.matmul(k[r, h][:, None], X)[:, 0])
            X = X + k[r, h][:, :, None] * new[:, None, :]
            S[at] = X
            o[r, h] = torch.matmul(q[r, h][:, None], X)[:, 0] / math.sqrt(d)
        out[st["idx_out"].long(), h] = S
    return o, out
