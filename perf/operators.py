"""The operators between the QKV projection and the output projection of a served decoder layer, as workloads.

Three operators that follow one another in every step of a serving loop over a paged key/value cache:

  slots   pages for the new tokens of every request, their slots in the cache and their positions, from the
          requests' lengths (once per step);
  rope    the norms of the query and key heads, the rotation by position (one axis or several) and the write of
          keys and values into the cache, from the QKV projection's output (once per layer);
  attn    attention of the new tokens over the cache, in which groups of requests share a long prefix that lies
          in the cache once (once per layer).

`run` computes them in their plain form, or, where `own` is true, with the library's entry points.  Shapes are
those of the QKV projections this repository works with (32 query heads with 8 or 4 key/value heads of 128
channels) and generic ones around them.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda"
BF16, F32, F64, I32 = torch.bfloat16, torch.float32, torch.float64, torch.int32


# ------------------------------------------------------------------------------------------------ lengths

def _ragged(total: int, n: int, lo: int, rng: random.Random) -> list:
    """n whole numbers of at least lo with the given sum, unequal as the lengths of real requests are."""
    if n == 0:
        return []
    free = total - lo * n
    assert free >= 0
    w = [rng.random() ** 2 + 0.05 for _ in range(n)]
    s = sum(w)
    out = [lo + int(free * x / s) for x in w]
    i = 0
    while sum(out) < total:
        out[i % n] += 1
        i += 1
    return out


def _lengths(case):
    """(new tokens, tokens in the cache before them) of every request."""
    rng = random.Random(case["lens"])
    R, T = case["R"], case["T"]
    if case["kind"] == "decode":          # one new token each
        assert T == R
        new = [1] * R
    elif case["kind"] == "mixed":         # most requests with one token, every seventh with a piece of its prompt
        big = [r for r in range(R) if r % 7 == 3 or R < 7]
        new = [1] * R
        for r, x in zip(big, _ragged(T - (R - len(big)), len(big), 1, rng)):
            new[r] = x
    else:                                 # "prompt": pieces of prompts
        new = _ragged(T, R, 0, rng)
    old = _ragged(case["old"], R, 0, rng)
    return new, old


def _groups(case):
    """First request of every group with a shared prefix, and the prefix lengths."""
    P, R = case["groups"], case["R"]
    off = [R * g // P for g in range(P + 1)] if P else [0]
    rng = random.Random(case["lens"] + 1)
    return off, (_ragged(case["prefix"], P, 0, rng) if P else [])


# ------------------------------------------------------------------------------------------------ the cases

def listed():
    return [
        # a few chats answering at once: one new token each, the smallest call of a decoding step
        dict(name="slots_decode_16", op="slots", kind="decode", R=16, T=16, old=11000, page=16, lens=1),
        # a full server: a thousand requests with one new token each
        dict(name="slots_decode_1024", op="slots", kind="decode", R=1024, T=1024, old=1500000, page=32, lens=2),
        # a step that mixes running requests with pieces of new prompts
        dict(name="slots_mixed_16400", op="slots", kind="mixed", R=211, T=16400, old=300000, page=64, lens=3),
        # one token of one request, where only latency counts
        dict(name="rope_1", op="rope", T=1, Hq=32, Hk=8, D=128, rot=128, axes=1, inter=False, pos=40000, page=16),
        # a decoding step of 256 requests
        dict(name="rope_256", op="rope", T=256, Hq=32, Hk=8, D=128, rot=128, axes=1, inter=False, pos=130000, page=64),
        # a prompt of 8192 tokens
        dict(name="rope_8192", op="rope", T=8192, Hq=32, Hk=8, D=128, rot=128, axes=1, inter=False, pos=8192, page=64),
        # image and video tokens with time, height and width positions, odd count
        dict(name="rope_axes_5001", op="rope", T=5001, Hq=32, Hk=4, D=128, rot=128, axes=3, inter=False, pos=2000, page=16),
        # one chat, one new token over six hundred cached ones: the smallest call
        dict(name="attn_single_600", op="attn", kind="decode", R=1, T=1, old=600, Hq=32, Hk=8, D=128, page=16, groups=0,
             prefix=0, lens=4),
        # 32 chats behind one system prompt of 4096 tokens
        dict(name="attn_shared_32", op="attn", kind="decode", R=32, T=32, old=14500, Hq=32, Hk=8, D=128, page=16, groups=1,
             prefix=4096, lens=5),
        # 256 requests over one long document of 16384 tokens
        dict(name="attn_shared_256", op="attn", kind="decode", R=256, T=256, old=131000, Hq=32, Hk=8, D=128, page=64, groups=1,
             prefix=16384, lens=6),
        # seven long contexts with nothing in common
        dict(name="attn_long_7", op="attn", kind="decode", R=7, T=7, old=207001, Hq=32, Hk=4, D=128, page=128, groups=0,
             prefix=0, lens=7),
        # prompts of six requests behind a shared prefix of 2048 tokens, computed in one step
        dict(name="attn_prompts_8001", op="attn", kind="prompt", R=6, T=8001, old=3001, Hq=32, Hk=8, D=128, page=64, groups=1,
             prefix=2048, lens=8),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    cap_b = {o: max(work(c)["bytes"] for c in listed() if c["op"] == o) for o in ("slots", "rope", "attn")}
    cap_f = {o: max(work(c)["flops"] for c in listed() if c["op"] == o) for o in ("slots", "rope", "attn")}
    op = rng.choice(["slots", "rope", "attn", "attn"])
    while True:
        if op == "slots":
            kind = rng.choice(["decode", "mixed", "prompt"])
            R = _log(rng, 1, 1024)
            T = R if kind == "decode" else R + _log(rng, 1, 15000)
            c = dict(op=op, kind=kind, R=R, T=T, old=R * _log(rng, 1, 1400), page=rng.choice([16, 32, 64, 128]),
                     lens=rng.randrange(1 << 20))
        elif op == "rope":
            Hk = rng.choice([1, 2, 4, 8])
            D = rng.choice([64, 128])
            c = dict(op=op, T=_log(rng, 1, 8192), Hq=Hk * rng.choice([1, 2, 4, 5, 7, 8]), Hk=Hk, D=D,
                     rot=rng.choice([D, D, D // 2]), axes=rng.choice([1, 1, 2, 3]), inter=rng.random() < 0.3,
                     pos=_log(rng, 1000, 1000000), page=rng.choice([16, 32, 64, 128]))
        else:
            Hk = rng.choice([1, 2, 4, 8])
            kind = rng.choice(["decode", "decode", "mixed", "prompt"])
            R = _log(rng, 1, 256 if kind == "decode" else 16)
            T = R if kind == "decode" else R + _log(rng, 1, 4000)
            groups = rng.choice([0, 1, 1, min(3, R)])
            c = dict(op=op, kind=kind, R=R, T=T, old=R * _log(rng, 1, 4000), Hq=Hk * rng.choice([1, 2, 4, 5, 7, 8, 16]), Hk=Hk,
                     D=rng.choice([64, 128, 128]), page=rng.choice([16, 32, 64, 128]), groups=groups,
                     prefix=_log(rng, 1, 16384) * groups, lens=rng.randrange(1 << 20))
            if T * c["Hq"] * max(c["prefix"], 1) > 600e6:      # the plain form holds all scores of a prefix
                continue
        w = work(c)
        if w["bytes"] <= cap_b[op] and w["flops"] <= cap_f[op]:
            return c


def work(case):
    """What one pass cannot do without."""
    if case["op"] == "slots":
        R, T = case["R"], case["T"]
        new, old = _lengths(case)
        p = case["page"]
        grown = sum((o + n + p - 1) // p - (o + p - 1) // p for n, o in zip(new, old))
        # lengths and first positions; row offsets, lengths after the step; slots and positions; a page number read for
        # every page the tokens touch, one written for every page taken
        touched = sum((o + n - 1) // p - o // p + 1 for n, o in zip(new, old) if n)
        return {"bytes": 4 * (3 * R) + 4 * (2 * R + 1) + 8 * T + 4 * (touched + grown), "flops": 0}
    if case["op"] == "rope":
        T, Hq, Hk, D = case["T"], case["Hq"], case["Hk"], case["D"]
        b = 2 * T * (Hq + 2 * Hk) * D * 2 + T * 4 * (case["axes"] + 1) + 2 * D * 2 + case["rot"] * 2
        return {"bytes": b, "flops": T * (Hq + Hk) * (3 * D + 4 * D) + T * case["rot"] * 10}
    new, old = _lengths(case)
    off, pre = _groups(case)
    Hq, Hk, D = case["Hq"], case["Hk"], case["D"]
    keys = sum(o + n for n, o in zip(new, old) if n) + sum(pre)
    pairs = sum(n * o + n * (n + 1) // 2 for n, o in zip(new, old))
    for g, p in enumerate(pre):
        pairs += p * sum(new[off[g]:off[g + 1]])
    T = case["T"]
    return {"bytes": keys * Hk * D * 4 + 2 * T * Hq * D * 2 + T * Hq * 4, "flops": 4 * pairs * Hq * D}


# ------------------------------------------------------------------------------------------------ inputs

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed) & 0x7FFFFFFF)


def _randn(shape, g, mul=1.0):
    return (torch.randn(shape, generator=g, device=DEV, dtype=F32) * mul).to(BF16)


def _i32(x):
    return torch.tensor(x, dtype=I32, device=DEV)


def _inv_freq(rot):
    return (1.0 / 1000000.0 ** (torch.arange(0, rot, 2, dtype=F64) / rot)).to(F32).to(DEV)


def prepare(case, seed):
    return {"slots": _prepare_slots, "rope": _prepare_rope, "attn": _prepare_attn}[case["op"]](case, seed)


def _prepare_slots(case, seed):
    g = _gen(seed)
    new, old = _lengths(case)
    R, T, p = case["R"], case["T"], case["page"]
    order = torch.randperm(R, generator=g, device=DEV)
    new_t, old_t = _i32(new)[order].contiguous(), _i32(old)[order].contiguous()
    cols = max((n + o + p - 1) // p for n, o in zip(new, old)) + 2
    n_old = sum((o + p - 1) // p for o in old)
    n_free = sum((n + o + p - 1) // p for n, o in zip(new, old)) - n_old + 5
    pages = torch.randperm(n_old + n_free, generator=g, device=DEV).to(I32)
    table = torch.full((R, cols), -1, dtype=I32, device=DEV)
    have = (old_t + p - 1) // p
    col = torch.arange(cols, device=DEV, dtype=I32)[None]
    held = col < have[:, None]
    table[held] = pages[:n_old]
    s = dict(op="slots", case=case, new=new_t, old=old_t, base=torch.randint(0, 5000, (R,), generator=g, device=DEV, dtype=I32),
             free=pages[n_old:].contiguous(), table=table, T=T, page=p)
    s["row_off"] = torch.empty(R + 1, dtype=I32, device=DEV)
    s["kv_len"] = torch.empty(R, dtype=I32, device=DEV)
    s["slots"] = torch.empty(T, dtype=I32, device=DEV)
    s["pos"] = torch.empty(T, dtype=I32, device=DEV)
    s["taken"] = torch.empty(1, dtype=I32, device=DEV)
    return s


def _prepare_rope(case, seed):
    g = _gen(seed)
    T, Hq, Hk, D, rot, axes, page = (case[k] for k in ("T", "Hq", "Hk", "D", "rot", "axes", "page"))
    n_pages = (T + T // 4 + page) // page
    s = dict(op="rope", case=case, Hq=Hq, Hk=Hk, D=D, rot=rot, inter=case["inter"])
    s["qkv"] = _randn((T, (Hq + 2 * Hk) * D), g, 1.5)
    s["gq"] = (torch.rand(D, generator=g, device=DEV) + 0.5).to(BF16)
    s["gk"] = (torch.rand(D, generator=g, device=DEV) + 0.5).to(BF16)
    s["eps"] = 1e-6
    s["inv"] = _inv_freq(rot)
    s["pos"] = torch.randint(0, case["pos"], (axes, T), generator=g, device=DEV, dtype=I32)
    if axes > 1:      # a quarter of the pairs turns by the first axis, the rest is shared out among the others
        n = rot // 2
        a = [0] * (n // 4)
        rest = n - n // 4
        for i in range(1, axes):
            a += [i] * (rest * i // (axes - 1) - rest * (i - 1) // (axes - 1))
        s["axis"] = torch.tensor(a, dtype=torch.uint8, device=DEV)
    else:
        s["axis"] = None
    slots = torch.randperm(n_pages * page, generator=g, device=DEV)[:T].to(I32)
    pad = T // 50     # the last rows only fill a captured step up: they have no slot
    if pad:
        slots[T - pad:] = -1
    s["slots"] = slots.contiguous()
    # one page more than the cache has, for the plain form's rows without a slot
    s["k_store"] = torch.zeros(n_pages + 1, page, Hk, D, dtype=BF16, device=DEV)
    s["v_store"] = torch.zeros(n_pages + 1, page, Hk, D, dtype=BF16, device=DEV)
    s["k"], s["v"] = s["k_store"][:n_pages], s["v_store"][:n_pages]
    s["q"] = torch.empty(T, Hq * D, dtype=BF16, device=DEV)
    if own:
        from paper_2604_12782_b200 import binding as B
        s["cache"] = B.KvCache(s["k"], s["v"])
        s["rope"] = B.Rope(s["inv"], axis=s["axis"], interleaved=s["inter"])
    return s


def _prepare_attn(case, seed):
    g = _gen(seed)
    new, old = _lengths(case)
    off, pre = _groups(case)
    R, T, Hq, Hk, D, p = (case[k] for k in ("R", "T", "Hq", "Hk", "D", "page"))
    kv = [n + o for n, o in zip(new, old)]
    np_own = [(x + p - 1) // p for x in kv]
    np_pre = [(x + p - 1) // p for x in pre]
    n_pages = sum(np_own) + sum(np_pre) + 3
    pages = torch.randperm(n_pages, generator=g, device=DEV).to(I32)

    def tables(counts, start):
        t = torch.full((max(len(counts), 1), max(counts + [1])), -1, dtype=I32, device=DEV)
        for i, c in enumerate(counts):
            t[i, :c] = pages[start:start + c]
            start += c
        return t, start
    s = dict(op="attn", case=case, Hq=Hq, Hk=Hk, D=D, page=p, new=new, kv=kv, groups=off, pre=pre)
    s["table"], at = tables(np_own, 0)
    s["ptable"], _ = tables(np_pre, at)
    s["k"] = _randn((n_pages, p, Hk, D), g)
    s["v"] = _randn((n_pages, p, Hk, D), g)
    s["q"] = _randn((T, Hq * D), g, 2.0)
    row = [0]
    for n in new:
        row.append(row[-1] + n)
    s["rows"] = row
    s["row_off"], s["kv_len"] = _i32(row), _i32(kv)
    s["group_off"], s["prefix_len"] = (_i32(off), _i32(pre)) if pre else (None, None)
    s["scale"] = 1.0 / math.sqrt(D)
    s["o"] = torch.empty(T, Hq * D, dtype=BF16, device=DEV)
    s["lse"] = torch.empty(T, Hq, dtype=F32, device=DEV)
    if own:
        from paper_2604_12782_b200 import binding as B
        s["cache"] = B.KvCache(s["k"], s["v"])
        s["max_new"] = max(new)
        n = B.osc_paged_attention_workspace_bytes(T, Hq, D, R, len(pre))
        s["ws"] = torch.empty(n, dtype=torch.uint8, device=DEV)
    return s


# ------------------------------------------------------------------------------------------------ one pass

def run(state):
    return {"slots": _run_slots, "rope": _run_rope, "attn": _run_attn}[state["op"]](state)


def _run_slots(s):
    if own:
        from paper_2604_12782_b200 import binding as B
        B.osc_kv_slots(s["old"], s["new"], s["base"], s["page"], s["free"], s["table"], s["row_off"], s["kv_len"],
                       s["slots"], s["pos"], s["taken"])
        return s["row_off"], s["kv_len"], s["table"], s["slots"], s["pos"], s["taken"]
    p, table, free = s["page"], s["table"], s["free"]
    old, new = s["old"].long(), s["new"].long()
    R, cols = table.shape
    row_off = torch.zeros(R + 1, dtype=torch.long, device=DEV)
    row_off[1:] = torch.cumsum(new, 0)
    kv = old + new
    have, want = (old + p - 1) // p, (kv + p - 1) // p
    need = want - have
    first = torch.cumsum(need, 0) - need
    col = torch.arange(cols, device=DEV)[None]
    src = first[:, None] + col - have[:, None]
    fresh = (col >= have[:, None]) & (col < want[:, None])
    page = torch.where(src < free.numel(), free[src.clamp(0, free.numel() - 1)], -1)
    table.copy_(torch.where(fresh, page, table))
    t = torch.arange(s["T"], device=DEV)
    r = torch.searchsorted(row_off[1:], t, right=True).clamp(max=R - 1)
    at = old[r] + t - row_off[r]
    pg = table[r, (at // p).clamp(0, cols - 1)].long()
    live = t < row_off[R]
    slots = torch.where(live & (pg >= 0), pg * p + at % p, -1)
    pos = torch.where(live, s["base"][r] + at, 0)
    return (row_off.to(I32), kv.to(I32), table, slots.to(I32), pos.to(I32), need.sum().to(I32).reshape(1))


def _run_rope(s):
    if own:
        from paper_2604_12782_b200 import binding as B
        B.osc_qk_norm_rope(s["qkv"], s["Hq"], s["cache"], s["q"], s["pos"], s["rope"], gamma_q=s["gq"], gamma_k=s["gk"],
                           eps=s["eps"], slots=s["slots"])
        return s["q"], s["k"], s["v"]
    T, Hq, Hk, D, rot = s["qkv"].shape[0], s["Hq"], s["Hk"], s["D"], s["rot"]
    x = s["qkv"].view(T, Hq + 2 * Hk, D).float()
    n = rot // 2
    pos = s["pos"].double()
    ang = (pos[s["axis"].long()].T if s["axis"] is not None else pos[0][:, None]) * s["inv"].double()[None]
    cos, sin = torch.cos(ang).float()[:, None], torch.sin(ang).float()[:, None]

    def turn(h, gamma):
        h = h * torch.rsqrt((h * h).mean(-1, keepdim=True) + s["eps"]) * gamma.float()
        if s["inter"]:
            a, b = h[..., 0:rot:2], h[..., 1:rot:2]
            r = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
        else:
            a, b = h[..., :n], h[..., n:rot]
            r = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
        return torch.cat((r, h[..., rot:]), -1).to(BF16)
    q = turn(x[:, :Hq], s["gq"])
    k = turn(x[:, Hq:Hq + Hk], s["gk"])
    v = s["qkv"].view(T, Hq + 2 * Hk, D)[:, Hq + Hk:]
    spare = s["k"].shape[0] * s["k"].shape[1]
    to = torch.where(s["slots"] >= 0, s["slots"].long(), spare)
    s["k_store"].view(-1, Hk, D)[to] = k
    s["v_store"].view(-1, Hk, D)[to] = v
    return q.reshape(T, Hq * D), s["k"], s["v"]


def _run_attn(s):
    if own:
        from paper_2604_12782_b200 import binding as B
        B.osc_paged_attention(s["q"], s["cache"], s["row_off"], s["kv_len"], s["table"], s["o"], s["ws"], s["scale"],
                              lse=s["lse"], group_off=s["group_off"], prefix_len=s["prefix_len"],
                              prefix_table=s["ptable"] if s["pre"] else None, max_new=s["max_new"])
        return s["o"], s["lse"]
    Hq, Hk, D, p = s["Hq"], s["Hk"], s["D"], s["page"]
    G, T = Hq // Hk, s["q"].shape[0]
    q = s["q"].view(T, Hk, G, D).float() * s["scale"]
    out = torch.zeros(T, Hk, G, D, device=DEV)
    lse = torch.zeros(T, Hk, G, device=DEV)

    def gather(store, row, n):
        return store[row[:(n + p - 1) // p].long()].reshape(-1, Hk, D)[:n].float()
    off, pre = (s["groups"], s["pre"]) if s["pre"] else ([0, len(s["new"])], [0])
    for g, np_ in enumerate(pre):
        a, b = s["rows"][off[g]], s["rows"][off[g + 1]]
        if a == b:
            continue
        # the shared prefix, for all rows of the group at once
        if np_:
            kp, vp = gather(s["k"], s["ptable"][g], np_), gather(s["v"], s["ptable"][g], np_)
            sp = torch.einsum("thgd,khd->thgk", q[a:b], kp)
            mp = sp.amax(-1)
        else:
            mp = torch.full((b - a, Hk, G), -math.inf, device=DEV)
        m, own_part = mp.clone(), []
        for r in range(off[g], off[g + 1]):
            n, kv, t0 = s["new"][r], s["kv"][r], s["rows"][r]
            if not n:
                continue
            ko, vo = gather(s["k"], s["table"][r], kv), gather(s["v"], s["table"][r], kv)
            so = torch.einsum("thgd,khd->thgk", q[t0:t0 + n], ko)
            if n > 1:
                seen = torch.arange(kv, device=DEV)[None] <= kv - n + torch.arange(n, device=DEV)[:, None]
                so.masked_fill_(~seen[:, None, None], -math.inf)
            i = slice(t0 - a, t0 - a + n)
            m[i] = torch.maximum(m[i], so.amax(-1))
            own_part.append((i, so, vo))
        l, acc = torch.zeros_like(m), torch.zeros(b - a, Hk, G, D, device=DEV)
        if np_:
            e = sp.sub_(m[..., None]).exp_()
            l += e.sum(-1)
            acc += torch.einsum("thgk,khd->thgd", e, vp)
        for i, so, vo in own_part:
            e = so.sub_(m[i][..., None]).exp_()
            l[i] += e.sum(-1)
            acc[i] += torch.einsum("thgk,khd->thgd", e, vo)
        out[a:b] = acc / l[..., None]
        lse[a:b] = m + torch.log(l)
    return out.to(BF16).view(T, Hq * D), lse.view(T, Hq)


# ------------------------------------------------------------------------------------------------ 64 bits

def exact(case, seed):
    if case["op"] == "slots":
        return None
    s = prepare(case, seed)
    Hq, Hk, D = s["Hq"], s["Hk"], s["D"]
    if case["op"] == "rope":
        T, rot = s["qkv"].shape[0], s["rot"]
        heads = s["qkv"].double().view(T, Hq + 2 * Hk, D)
        which = s["axis"].long() if s["axis"] is not None else torch.zeros(rot // 2, dtype=torch.long, device=DEV)
        angle = s["pos"].double()[which] * s["inv"].double()[:, None]          # [pair, token]
        i = torch.arange(rot // 2, device=DEV)
        first, second = (2 * i, 2 * i + 1) if s["inter"] else (i, i + rot // 2)

        def one(h, gamma):                                                     # [token, head, channel]
            y = h / torch.sqrt(h.pow(2).sum(-1, keepdim=True) / D + s["eps"]) * gamma.double()
            z = torch.complex(y[..., first], y[..., second]) * torch.polar(torch.ones_like(angle), angle).T[:, None]
            y = y.clone()
            y[..., first], y[..., second] = z.real, z.imag
            return y
        k = torch.zeros(s["k"].shape, dtype=F64, device=DEV).view(-1, Hk, D)
        v = torch.zeros(s["v"].shape, dtype=F64, device=DEV).view(-1, Hk, D)
        live = s["slots"] >= 0
        to = s["slots"][live].long()
        k[to] = one(heads[:, Hq:Hq + Hk], s["gk"])[live]
        v[to] = heads[:, Hq + Hk:][live]
        return one(heads[:, :Hq], s["gq"]).reshape(T, Hq * D), k.view(s["k"].shape), v.view(s["v"].shape)
    if work(case)["flops"] > 6e11:
        return None
    T, p, G = s["q"].shape[0], s["page"], Hq // Hk
    out = torch.zeros(T, Hq, D, dtype=F64, device=DEV)
    lse = torch.full((T, Hq), -math.inf, dtype=F64, device=DEV)
    q = s["q"].double().view(T, Hq, D)
    group = {}
    for g in range(len(s["pre"])):
        for r in range(s["groups"][g], s["groups"][g + 1]):
            group[r] = g
    for r, (n, kv) in enumerate(zip(s["new"], s["kv"])):
        t0 = s["rows"][r]
        if not n:
            continue
        key, val, shared = [], [], 0
        if r in group:
            shared = s["pre"][group[r]]
            pages = s["ptable"][group[r]].long()
            j = torch.arange(shared, device=DEV)
            key.append(s["k"][pages[j // p], j % p])
            val.append(s["v"][pages[j // p], j % p])
        j = torch.arange(kv, device=DEV)
        pages = s["table"][r].long()
        key.append(s["k"][pages[j // p], j % p])
        val.append(s["v"][pages[j // p], j % p])
        key, val = torch.cat(key), torch.cat(val)
        at = torch.arange(shared + kv, device=DEV)
        for h in range(Hk):
            kd, vd = key[:, h].double(), val[:, h].double()
            for a in range(0, n, 512):
                b = min(n, a + 512)
                qi = q[t0 + a:t0 + b, h * G:(h + 1) * G]
                sc = (qi.reshape(-1, D) @ kd.T).view(b - a, G, -1) * s["scale"]
                limit = shared + kv - n + torch.arange(a, b, device=DEV)
                sc.masked_fill_((at[None] > limit[:, None])[:, None], -math.inf)
                z = torch.logsumexp(sc, -1)
                lse[t0 + a:t0 + b, h * G:(h + 1) * G] = z
                out[t0 + a:t0 + b, h * G:(h + 1) * G] = (torch.exp(sc - z[..., None]).view(-1, sc.shape[-1]) @ vd).view(b - a, G, D)
    return out.view(T, Hq * D), lse
