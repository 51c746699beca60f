"""Decoding with more than one continuation of a request over a paged key/value cache, as workloads.

Five calls that a serving loop makes when it drafts trees of tokens and verifies them in one step, or keeps several
beams of a request:

  mask      which drafted tokens each drafted token descends from (a bit mask) and their positions, from the tokens'
            parents (once per step);
  attn      attention of the drafted trees over the cache: the keys of a request's context, and of a token's own
            ancestors (once per layer);
  logprobs  log probabilities of given tokens, log-sum-exp, entropy and the best alternatives, from rows of logits
            (once per step);
  compact   the keys and values of the accepted tokens moved together behind the context, in all layers (once per
            step);
  reorder   pages of dead beams given back, rows of the page table forked from the beams that go on, and the pages
            that are only partly filled copied, in all layers (once per step).

`run` computes them in their plain form, or, where `own` is true, with the library's entry points.  Head counts are
those of the QKV projections this repository works with (32 query heads with 8 or 4 key/value heads of 128 channels)
and generic ones around them.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda"
BF16, F32, F64, I32, I64 = torch.bfloat16, torch.float32, torch.float64, torch.int32, torch.int64


# ------------------------------------------------------------------------------------------------ lengths

def _ragged(total: int, n: int, lo: int, rng: random.Random) -> list:
    """n whole numbers of at least lo with the given sum, unequal as the lengths of real requests are."""
    if n == 0:
        return []
    free = total - lo * n
    assert free >= 0
    w = [rng.random() ** 2 + 0.15 for _ in range(n)]
    s = sum(w)
    out = [lo + int(free * x / s) for x in w]
    for i in range(total - sum(out)):
        out[i % n] += 1
    return out


def _lengths(case):
    """(drafted tokens, tokens in the cache before them) of every request."""
    rng = random.Random(case["lens"])
    new = _ragged(case["T"], case["R"], 1, rng)
    return new, _ragged(case["old"], case["R"], 0, rng)


def _groups(case):
    """First request of every group with a shared prefix, and the prefix lengths."""
    P, R = case["groups"], case["R"]
    rng = random.Random(case["lens"] + 1)
    return [R * g // P for g in range(P + 1)] if P else [0], (_ragged(case["prefix"], P, 0, rng) if P else [])


def _parents(new, rng):
    """Parents of every request's tokens: a main chain with branches, as a drafting model leaves it, several roots among them."""
    out = []
    for n in new:
        for i in range(n):
            x = rng.random()
            out.append(i - 1 if i == 0 or x < 0.5 else -1 if x < 0.55 else rng.randrange(max(0, i - 12), i))
    return out


def _beams(case):
    """Tokens of every row of the table (beams of a request are equally long), and the forks of the step: (source, row)."""
    rng = random.Random(case["lens"])
    B, R = case["beams"], case["R"]
    lens, pairs = [], []
    for x in _ragged(case["old"], R // B, 1, rng):
        at = len(lens)
        dead = sorted(rng.sample(range(at, at + B), rng.randrange(1, B)))
        live = [i for i in range(at, at + B) if i not in dead]
        pairs += [(rng.choice(live), d) for d in dead]
        lens += [x] * B
    return lens, pairs


# ------------------------------------------------------------------------------------------------ the cases

def listed():
    return [
        # one chat whose next tokens are drafted as a small tree: the smallest call
        dict(name="mask_chat_26", op="mask", R=1, T=26, old=900, pad=0, words=1, lens=1),
        # a full server: 500 requests with trees of unequal sizes, filled up to a captured step's 16384 rows
        dict(name="mask_server_16201", op="mask", R=500, T=16201, old=400000, pad=183, words=4, lens=2),
        # the same chat in one layer of attention: latency
        dict(name="attn_chat_26", op="attn", R=1, T=26, old=900, pad=0, Hq=32, Hk=8, D=128, page=16, groups=0, prefix=0, words=1, lens=1),
        # two dozen requests of a few thousand tokens, trees of some forty tokens each
        dict(name="attn_trees_24", op="attn", R=24, T=1003, old=100300, pad=21, Hq=32, Hk=8, D=128, page=64, groups=0, prefix=0, words=4,
             lens=4),
        # forty chats behind one system prompt, with small trees (a dozen tokens)
        dict(name="attn_shared_40", op="attn", R=40, T=521, old=30011, pad=0, Hq=32, Hk=4, D=128, page=16, groups=1, prefix=4100, words=2,
             lens=5),
        # five long documents, large trees
        dict(name="attn_long_5", op="attn", R=5, T=317, old=200003, pad=3, Hq=32, Hk=8, D=128, page=128, groups=0, prefix=0, words=4, lens=6),
        # a step of 26 drafted tokens (a tree), three children of each looked up, fp32 logits
        dict(name="logprobs_26", op="logprobs", T=26, V=128000, masked=0, f32=True, ids=3, top=5, temperature=0.7),
        # a prompt of 3001 tokens scored against itself (perplexity of a quantized model), vocabulary filled up to a multiple of 256
        dict(name="logprobs_3001", op="logprobs", T=3001, V=152064, masked=395, f32=False, ids=1, top=20, temperature=1.0),
        # one chat: five of its 26 drafted tokens accepted, 36 layers
        dict(name="compact_chat", op="compact", L=36, R=1, T=26, old=900, Hk=8, D=128, page=16, most=5, lens=1),
        # 96 requests with trees of about fifty tokens, up to twelve of them accepted
        dict(name="compact_96", op="compact", L=36, R=96, T=4803, old=9600, Hk=8, D=128, page=64, most=12, lens=8),
        # one request with four beams
        dict(name="reorder_4", op="reorder", L=36, R=4, beams=4, old=777, Hk=8, D=128, page=16, lens=9),
        # two dozen requests with eight beams each
        dict(name="reorder_192", op="reorder", L=36, R=192, beams=8, old=14400, Hk=8, D=128, page=32, lens=10),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["mask", "attn", "attn", "logprobs", "compact", "reorder"])
    cap_b = max(work(c)["bytes"] for c in listed() if c["op"] == op)
    cap_f = max(work(c)["flops"] for c in listed() if c["op"] == op)
    while True:
        lens, page = rng.randrange(1 << 20), rng.choice([16, 32, 64, 128])
        R = _log(rng, 1, 500 if op == "mask" else 96)
        T = R + _log(rng, 1, 64) * R - rng.randrange(R)
        if op == "mask":
            c = dict(op=op, R=R, T=T, old=R * _log(rng, 1, 4000), pad=rng.choice([0, 0, _log(rng, 1, 200)]), words=rng.choice([1, 2, 4, 7]), lens=lens)
        elif op == "attn":
            Hk, groups = rng.choice([1, 2, 4, 8]), rng.choice([0, 0, 1, min(3, R)])
            c = dict(op=op, R=R, T=T, old=R * _log(rng, 1, 40000), pad=rng.choice([0, 0, _log(rng, 1, 50)]), Hq=Hk * rng.choice([1, 2, 4, 5, 7, 8, 16]),
                     Hk=Hk, D=rng.choice([64, 128, 128]), page=page, groups=groups, prefix=_log(rng, 1, 8192) * groups, words=0, lens=lens)
            new, old = _lengths(c)
            c["words"] = (max(new) + 31) // 32 + rng.choice([0, 0, 1])
            # the plain form holds all scores
            if R * max(new) * c["Hq"] * (max(x + n for x, n in zip(old, new)) + c["prefix"]) > 1.0e9:
                continue
        elif op == "logprobs":
            c = dict(op=op, T=_log(rng, 1, 3001), V=_log(rng, 1000, 262144), masked=0, f32=rng.random() < 0.4, ids=rng.choice([1, 1, 2, 5]),
                     top=rng.choice([0, 1, 5, 8, 20, 32]), temperature=rng.choice([1.0, 1.0, 0.6, 1.3]))
            c["masked"] = rng.choice([0, c["V"] // 50])
        elif op == "compact":
            c = dict(op=op, L=_log(rng, 1, 48), R=R, T=T, old=R * _log(rng, 1, 100), Hk=rng.choice([1, 2, 4, 8]), D=rng.choice([64, 128]), page=page,
                     most=rng.choice([1, 4, 8, 12]), lens=lens)
        else:
            B = rng.choice([2, 4, 8])
            n = _log(rng, 1, 24)
            c = dict(op=op, L=_log(rng, 1, 48), R=n * B, beams=B, old=n * _log(rng, 1, 700), Hk=rng.choice([1, 2, 4, 8]), D=rng.choice([64, 128]),
                     page=page, lens=lens)
        w = work(c)
        if 0 < w["bytes"] <= cap_b and w["flops"] <= cap_f:
            return c


def work(case):
    """What one pass cannot do without."""
    op = case["op"]
    if op == "mask":
        R, T = case["R"], case["T"] + case["pad"]
        return {"bytes": 4 * T * (2 + case["words"]) + 4 * (2 * R + 1), "flops": 0}
    if op == "attn":
        new, old = _lengths(case)
        off, pre = _groups(case)
        Hq, Hk, D, T = case["Hq"], case["Hk"], case["D"], case["T"]
        pairs = sum(n * (o + 1) for n, o in zip(new, old)) + sum(p * sum(new[off[g]:off[g + 1]]) for g, p in enumerate(pre))
        keys = sum(new) + sum(old) + sum(pre)
        return {"bytes": keys * Hk * D * 4 + 2 * T * Hq * D * 2 + T * Hq * 4 + T * case["words"] * 4, "flops": 4 * pairs * Hq * D}
    if op == "logprobs":
        T, V = case["T"], case["V"]
        return {"bytes": T * V * (4 if case["f32"] else 2) + T * (8 * case["ids"] + 8 * case["top"] + 8), "flops": 4 * T * V}
    row = case["L"] * 2 * case["Hk"] * case["D"] * 2          # bytes of a token in all layers
    if op == "compact":
        moved = sum(sum(i != d for d, i in enumerate(k)) for k in _kept(case, random.Random(case["lens"] + 2)))
        return {"bytes": 2 * moved * row + 4 * (4 * case["R"] + 1), "flops": 0}
    lens, pairs = _beams(case)
    p = case["page"]
    gone, full, part = sum(-(-lens[d] // p) for _, d in pairs), sum(lens[d] // p for _, d in pairs), sum(lens[d] % p for _, d in pairs)
    return {"bytes": 2 * part * row + 4 * (4 * gone + 4 * full + 8 * len(pairs)), "flops": 0}


# ------------------------------------------------------------------------------------------------ inputs

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed) & 0x7FFFFFFF)


def _randn(shape, g, mul=1.0):
    return (torch.randn(shape, generator=g, device=DEV, dtype=F32) * mul).to(BF16)


def _i32(x):
    return torch.tensor(x, dtype=I32, device=DEV)


def prepare(case, seed):
    return {"mask": _prepare_mask, "attn": _prepare_attn, "logprobs": _prepare_logprobs, "compact": _prepare_compact,
            "reorder": _prepare_reorder}[case["op"]](case, seed)


def _prepare_mask(case, seed):
    new, old = _lengths(case)
    T = case["T"] + case["pad"]
    rng = random.Random(seed)
    row = [0]
    for n in new:
        row.append(row[-1] + n)
    s = dict(op="mask", words=case["words"], longest=max(new))
    # rows behind the last request hold what an earlier step left there
    s["parents"] = _i32(_parents(new, rng) + [rng.randrange(-1, 50) for _ in range(case["pad"])])
    s["row_off"], s["base"] = _i32(row), _i32(old)
    s["mask"] = torch.empty(T, case["words"], dtype=I32, device=DEV)
    s["pos"] = torch.empty(T, dtype=I32, device=DEV)
    return s


def _prepare_attn(case, seed):
    g = _gen(seed)
    new, old = _lengths(case)
    off, pre = _groups(case)
    R, T, Hq, Hk, D, p = case["R"], case["T"] + case["pad"], case["Hq"], case["Hk"], case["D"], case["page"]
    kv = [n + o for n, o in zip(new, old)]
    np_own, np_pre = [-(-x // p) for x in kv], [-(-x // p) for x in pre]
    n_pages = sum(np_own) + sum(np_pre) + 3
    pages = torch.randperm(n_pages, generator=g, device=DEV).to(I32)

    def table(counts, start):
        t = torch.full((max(len(counts), 1), max(counts + [1])), -1, dtype=I32, device=DEV)
        for i, c in enumerate(counts):
            t[i, :c] = pages[start:start + c]
            start += c
        return t
    s = dict(op="attn", Hq=Hq, Hk=Hk, D=D, page=p, longest=max(new), keys=max(kv) + max(pre + [0]), words=case["words"])
    s["table"], s["ptable"] = table(np_own, 0), table(np_pre, sum(np_own))
    s["k"], s["v"] = _randn((n_pages, p, Hk, D), g), _randn((n_pages, p, Hk, D), g)
    s["q"] = _randn((T, Hq * D), g, 2.0)
    row = [0]
    for n in new:
        row.append(row[-1] + n)
    s["row_off"], s["kv_len"] = _i32(row), _i32(kv)
    s["group_off"], s["prefix_len"] = (_i32(off), _i32(pre)) if pre else (None, None)
    s["mask"] = torch.zeros(T, case["words"], dtype=I32, device=DEV)
    bits, _ = _trees(_i32(_parents(new, random.Random(seed))), s["row_off"], max(new))
    rows, there = _rows_of(s["row_off"], max(new))
    s["mask"][rows[there]] = _packed(bits, case["words"])[there]
    s["scale"] = 1.0 / math.sqrt(D)
    # rows behind the last request are left as they are
    s["o"] = torch.zeros(T, Hq * D, dtype=BF16, device=DEV)
    s["lse"] = torch.zeros(T, Hq, dtype=F32, device=DEV)
    if own:
        from paper_2604_12782_b200 import binding as B
        s["cache"] = B.KvCache(s["k"], s["v"])
        s["ws"] = torch.empty(B.osc_paged_attention_workspace_bytes(T, Hq, D, R, len(pre)), dtype=torch.uint8, device=DEV)
    return s


def _prepare_logprobs(case, seed):
    g = _gen(seed)
    T, V, n = case["T"], case["V"], case["ids"]
    real = V - case["masked"]
    x = torch.randn(T, V, generator=g, device=DEV, dtype=F32)
    x *= 1.0 + 2.0 * torch.rand(T, 1, generator=g, device=DEV)
    # from undecided rows to very sure ones: one token ahead of the others
    best = torch.randint(0, real, (T,), generator=g, device=DEV)
    x[torch.arange(T, device=DEV), best] += 20.0 * torch.rand(T, generator=g, device=DEV)
    if case["masked"]:
        x[:, real:] = -math.inf        # the end of a vocabulary that is filled up
    ids = torch.randint(0, real, (T, n), generator=g, device=DEV)
    ids[::2, 0] = best[::2]
    return dict(op="logprobs", x=x if case["f32"] else x.to(BF16), ids=ids.to(I32), scale=1.0 / case["temperature"], top=case["top"],
                logprob=torch.empty(T, n, dtype=F32, device=DEV), lse=torch.empty(T, dtype=F32, device=DEV), entropy=torch.empty(T, dtype=F32, device=DEV),
                top_ids=torch.empty(T, case["top"], dtype=I32, device=DEV) if case["top"] else None,
                top_logprobs=torch.empty(T, case["top"], dtype=F32, device=DEV) if case["top"] else None)


def _kept(case, rng):
    """Indices of every request's accepted tokens: the main chain, drafted first, for some steps, then a branch behind it."""
    new, _ = _lengths(case)
    out = []
    for n in new:
        m = rng.randrange(0, min(case["most"], n) + 1)
        c = rng.randrange(0, m + 1)
        out.append(list(range(c)) + sorted(rng.sample(range(m, n), m - c)) if n - m >= m - c else list(range(m)))
    return out


def _layers(L, n_pages, page, Hk, D, g):
    """Keys and values of all layers, in one buffer each."""
    k, v = (torch.empty(L, n_pages, page, Hk, D, dtype=BF16, device=DEV) for _ in range(2))
    return k.normal_(generator=g), v.normal_(generator=g)


def _handle(s):
    from paper_2604_12782_b200 import binding as B
    return B.KvLayers([B.KvCache(k, v) for k, v in zip(s["k"], s["v"])])


def _prepare_compact(case, seed):
    g = _gen(seed)
    new, old = _lengths(case)
    R, p = case["R"], case["page"]
    kv = [n + o for n, o in zip(new, old)]
    counts = [-(-x // p) for x in kv]
    n_pages = sum(counts) + 2
    pages = torch.randperm(n_pages, generator=g, device=DEV).to(I32)
    table = torch.full((R, max(counts)), -1, dtype=I32, device=DEV)
    at = 0
    for i, c in enumerate(counts):
        table[i, :c] = pages[at:at + c]
        at += c
    kept = _kept(case, random.Random(case["lens"] + 2))
    cols = max(case["most"], 1)
    row = [0]
    for n in new:
        row.append(row[-1] + n)
    s = dict(op="compact", page=p, table=table, row_off=_i32(row), kv_len=_i32(kv), keep=_i32([k + [-1] * (cols - len(k)) for k in kept]),
             n_keep=_i32([len(k) for k in kept]), new_len=torch.empty(R, dtype=I32, device=DEV))
    s["k"], s["v"] = _layers(case["L"], n_pages, p, case["Hk"], case["D"], g)
    if own:
        s["layers"] = _handle(s)
    return s


def _prepare_reorder(case, seed):
    g = _gen(seed)
    lens, pairs = _beams(case)
    R, p, B = case["R"], case["page"], case["beams"]
    # every beam of a request holds the same full pages and a last page of its own, if that is only partly filled
    full = [x // p for x in lens]
    n_pages = sum(full[::B]) + sum(x % p > 0 for x in lens) + 5
    pages = torch.randperm(n_pages, generator=g, device=DEV).tolist()
    at = sum(full[::B])
    tails = [0] * R
    # The pages that the dead beams give back are the ones that the forks take, so that every pass does the same work.
    for i in range(R):
        if lens[i] % p:
            tails[i] = pages[at]
            at += 1
    dead = [d for _, d in pairs]
    free = sorted(tails[d] for d in dead if lens[d] % p)
    for d, t in zip([d for d in dead if lens[d] % p], free):
        tails[d] = t
    rows, start = [], 0
    for i in range(R):
        rows.append(pages[start:start + full[i]] + ([tails[i]] if lens[i] % p else []))
        if i % B == B - 1:
            start += full[i]
    cols = max(len(r) for r in rows)
    n = len(pairs)
    s = dict(op="reorder", page=p, n_pages=n_pages, table=_i32([r + [-1] * (cols - len(r)) for r in rows]), len=_i32(lens),
             to=_i32([0 if i in set(dead) else x for i, x in enumerate(lens)]), src=_i32([a for a, _ in pairs]), dst=_i32(dead),
             free=_i32(free + pages[at:]))
    s["refs"] = torch.zeros(n_pages, dtype=I32, device=DEV)
    held = s["table"][s["table"] >= 0].long()
    s["refs"].scatter_add_(0, held, torch.ones_like(held, dtype=I32))
    s["freed"] = torch.full((n_pages,), -1, dtype=I32, device=DEV)
    s["n_freed"], s["taken"] = torch.empty(1, dtype=I32, device=DEV), torch.empty(1, dtype=I32, device=DEV)
    s["copy_from"], s["copy_to"], s["copy_used"] = (torch.empty(n, dtype=I32, device=DEV) for _ in range(3))
    s["k"], s["v"] = _layers(case["L"], n_pages, p, case["Hk"], case["D"], g)
    if own:
        s["layers"] = _handle(s)
    return s


# ------------------------------------------------------------------------------------------------ one pass

def run(state):
    return {"mask": _run_mask, "attn": _run_attn, "logprobs": _run_logprobs, "compact": _run_compact, "reorder": _run_reorder}[state["op"]](state)


def _rows_of(row_off, longest):
    """Rows [R, longest] of every request's tokens, and which of them there are."""
    j = torch.arange(longest, device=DEV)[None]
    r0, r1 = row_off[:-1, None].long(), row_off[1:, None].long()
    return torch.where(r0 + j < r1, r0 + j, 0), r0 + j < r1


def _trees(parents, row_off, longest):
    """bits [R, longest, longest]: token m is an ancestor of token i, or i itself; depths [R, longest], roots at 0."""
    rows, there = _rows_of(row_off, longest)
    i = torch.arange(longest, device=DEV)
    par = parents[rows].long()
    known = there & (par >= -1) & (par < i[None])
    up = (par[..., None] == i) & known[..., None]
    reach = (up | ((i[:, None] == i[None]) & known[..., None])).to(F32)
    # paths of up to 1, 2, 4, ... steps
    for _ in range(max(1, (longest - 1).bit_length())):
        reach = ((reach @ reach) > 0).to(F32)
    rooted = (reach @ (known & (par == -1)).to(F32)[..., None]) > 0      # a token whose line does not end in a root is not there
    bits = (reach > 0) & rooted
    return bits, torch.where(rooted[..., 0], bits.sum(-1) - 1, 0)


def _packed(bits, words):
    """bits [..., n] as int32 [..., words]."""
    n = bits.shape[-1]
    x = torch.zeros(*bits.shape[:-1], 32 * words, dtype=I64, device=DEV)
    x[..., :min(n, 32 * words)] = bits[..., :32 * words]
    x = (x.unflatten(-1, (words, 32)) << torch.arange(32, device=DEV)).sum(-1)
    return torch.where(x >= 1 << 31, x - (1 << 32), x).to(I32)


def _run_mask(s):
    if own:
        from paper_2604_12782_b200 import binding as B
        B.osc_tree_mask(s["parents"], s["row_off"], s["base"], s["mask"], s["pos"])
        return s["mask"], s["pos"]
    rows, there = _rows_of(s["row_off"], s["longest"])
    here = there & (torch.arange(s["longest"], device=DEV)[None] < 32 * s["words"])     # tokens that have no bit are not there
    bits, depth = _trees(torch.where(here, s["parents"][rows], -2).flatten(), torch.arange(rows.shape[0] + 1, device=DEV) * s["longest"], s["longest"])
    alive = bits.any(-1)
    T = s["parents"].numel()
    spare = torch.where(there, rows, T).flatten()        # padded places go to a row behind the last one
    mask = torch.zeros(T + 1, s["words"], dtype=I32, device=DEV)
    pos = torch.zeros(T + 1, dtype=I32, device=DEV)
    mask[spare] = _packed(bits, s["words"]).flatten(0, 1)
    pos[spare] = torch.where(alive, s["base"][:, None] + depth, 0).to(I32).flatten()
    return mask[:T], pos[:T]


def _run_attn(s):
    if own:
        from paper_2604_12782_b200 import binding as B
        B.osc_tree_attention(s["q"], s["cache"], s["row_off"], s["kv_len"], s["table"], s["mask"], s["o"], s["ws"], s["scale"], lse=s["lse"],
                             group_off=s["group_off"], prefix_len=s["prefix_len"], prefix_table=s["ptable"] if s["prefix_len"] is not None else None,
                             max_new=s["longest"])
        return s["o"], s["lse"]
    Hq, Hk, D, p, N, K = s["Hq"], s["Hk"], s["D"], s["page"], s["longest"], s["keys"]
    G, T, R = Hq // Hk, s["q"].shape[0], s["kv_len"].numel()
    rows, there = _rows_of(s["row_off"], N)
    n, kv = there.sum(1)[:, None], s["kv_len"].long()[:, None]
    j = torch.arange(K, device=DEV)[None]
    # keys of every request: those of its group's prefix, then its own
    if s["prefix_len"] is not None:
        r = torch.arange(R, device=DEV)
        g = (torch.searchsorted(s["group_off"].long(), r, right=True) - 1).clamp(0, s["prefix_len"].numel() - 1)
        pre = s["prefix_len"].long()[g][:, None]
        front = s["ptable"][g[:, None], (j // p).clamp(max=s["ptable"].shape[1] - 1)]
    else:
        pre, front = torch.zeros_like(kv), torch.zeros_like(j)
    at = torch.where(j < pre, j, j - pre)
    page = torch.where(j < pre, front, torch.gather(s["table"].expand(R, -1), 1, (at // p).clamp(max=s["table"].shape[1] - 1)))
    page = torch.where(j < pre + kv, page, 0).long()
    keys = s["k"][page, at % p].permute(0, 2, 1, 3).float()               # [R, Hk, K, D]
    vals = s["v"][page, at % p].permute(0, 2, 1, 3).float()
    # what a row sees: the context, and among the new tokens those whose bits are set
    m = j - (pre + kv - n)                                                # [R, K]
    word = torch.gather(s["mask"][rows], 2, (m // 32).clamp(0, s["words"] - 1)[:, None].expand(-1, N, -1))
    bit = ((word >> (m % 32)[:, None]) & 1).bool() & (m < 32 * s["words"])[:, None]
    sees = ((m < 0)[:, None] | (bit & (m < n)[:, None])) & (j < pre + kv)[:, None]
    q = s["q"][rows].view(R, N, Hk, G, D).permute(0, 2, 1, 3, 4).reshape(R, Hk, N * G, D).float() * s["scale"]
    sc = (q @ keys.transpose(2, 3)).view(R, Hk, N, G, K)
    sc.masked_fill_(~sees[:, None, :, None], -math.inf)
    top = sc.amax(-1, keepdim=True)
    e = sc.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    l = e.sum(-1, keepdim=True)
    out = (e.view(R, Hk, N * G, K) @ vals).view(R, Hk, N, G, D) / torch.where(l > 0, l, 1.0)
    lse = (top + torch.log(l))[..., 0]
    # rows behind the last request stay 0
    o = torch.zeros(T, Hq * D, dtype=BF16, device=DEV)
    ls = torch.zeros(T, Hq, dtype=F32, device=DEV)
    o[rows[there]] = out.permute(0, 2, 1, 3, 4).reshape(R, N, Hq * D)[there].to(BF16)
    ls[rows[there]] = lse.permute(0, 2, 1, 3).reshape(R, N, Hq)[there]
    return o, ls


def _run_logprobs(s):
    if own:
        from paper_2604_12782_b200 import binding as B
        B.osc_token_logprobs(s["x"], s["ids"], s["logprob"], scale=s["scale"], lse=s["lse"], entropy=s["entropy"], top_ids=s["top_ids"],
                             top_logprobs=s["top_logprobs"])
        return {k: s[k] for k in ("logprob", "lse", "entropy", "top_ids", "top_logprobs")}
    x = s["x"]
    V, k = x.shape[1], s["top"]
    y = x.float() * s["scale"]
    top = y.amax(-1, keepdim=True)
    y -= top
    e = torch.exp(y)
    l = e.sum(-1, keepdim=True)
    ln = torch.log(l)
    entropy = ln - torch.where(e > 0, e * y, 0.0).sum(-1, keepdim=True) / l
    logprob = torch.gather(y, 1, s["ids"].long()) - ln
    out = dict(logprob=logprob, lse=(top + ln)[:, 0], entropy=entropy[:, 0], top_ids=None, top_logprobs=None)
    if k:
        # one whole number that orders by value, then by the lower index
        b = x.view(torch.int16).to(I32) << 16 if x.dtype == BF16 else x.view(I32)
        key = torch.where(b < 0, (b & 0x7FFFFFFF).neg_(), b).to(I64).mul_(1 << 32).sub_(torch.arange(V, device=DEV))
        top_ids = (-torch.topk(key, k, dim=1).values) % (1 << 32)
        out["top_ids"], out["top_logprobs"] = top_ids.to(I32), torch.gather(y, 1, top_ids) - ln
    return out


def _run_compact(s):
    if own:
        from paper_2604_12782_b200 import binding as B
        B.osc_kv_compact(s["layers"], s["row_off"], s["kv_len"], s["table"], s["keep"], s["n_keep"], s["new_len"])
        return s["k"], s["v"], s["new_len"]
    p, keep = s["page"], s["keep"].long()
    n = (s["row_off"][1:] - s["row_off"][:-1]).long()[:, None]
    d = torch.arange(keep.shape[1], device=DEV)[None]
    before = torch.cat((torch.full_like(keep[:, :1], -1), keep[:, :-1]), 1)
    good = ((d < s["n_keep"][:, None]) & (keep > before) & (keep < n)).cumprod(1).bool()
    ctx = s["kv_len"].long()[:, None] - n

    def slot(at):
        return torch.gather(s["table"], 1, at.clamp(0, s["table"].shape[1] * p - 1) // p).long() * p + at % p
    a, b = slot(ctx + keep)[good], slot(ctx + d)[good]
    for x in (s["k"], s["v"]):
        flat = x.flatten(1, 2)
        flat[:, b] = flat[:, a]
    return s["k"], s["v"], (ctx[:, 0] + good.sum(1)).to(I32)


def _run_reorder(s):
    if own:
        from paper_2604_12782_b200 import binding as B
        B.osc_kv_trim(s["len"], s["to"], s["page"], s["table"], s["refs"], s["freed"], s["n_freed"])
        B.osc_kv_fork(s["src"], s["dst"], s["len"], s["page"], s["free"], s["table"], s["refs"], s["copy_from"], s["copy_to"], s["copy_used"], s["taken"])
        B.osc_kv_copy_pages(s["layers"], s["copy_from"], s["copy_to"], s["copy_used"])
        return tuple(s[k] for k in ("k", "v", "table", "refs", "len", "freed", "n_freed", "copy_from", "copy_to", "copy_used", "taken"))
    p, table, refs, NP = s["page"], s["table"], s["refs"], s["n_pages"]
    col = torch.arange(table.shape[1], device=DEV)[None]
    # pages given back
    a, b = (s["to"] + p - 1) // p, (s["len"] + p - 1) // p
    gone = (col >= a[:, None]) & (col < b[:, None]) & (table >= 0)
    less = torch.zeros(NP + 1, dtype=I32, device=DEV).scatter_add_(0, torch.where(gone, table, NP).flatten().long(), gone.flatten().to(I32))[:NP]
    freed = (refs > 0) & (less >= refs)
    refs.copy_((refs - less).clamp(min=0))
    table.masked_fill_(gone, -1)
    order = torch.where(freed, torch.arange(NP, device=DEV), NP).sort().values
    s["freed"].copy_(torch.where(order < NP, order, s["freed"]))
    n_freed = freed.sum().to(I32)[None]
    # rows forked
    src, dst = s["src"].long(), s["dst"].long()
    ln = s["len"][src]
    full, used = ln // p, ln % p
    need = (used > 0).long()
    first = need.cumsum(0) - need
    new = torch.where(first < s["free"].numel(), s["free"][first.clamp(max=s["free"].numel() - 1)], -1)
    old = table[src]
    shared = col < full[:, None]
    tail = (col == full[:, None]) & (used > 0)[:, None]
    table[dst] = torch.where(shared, old, torch.where(tail, new[:, None], table[dst]))
    more = torch.cat((torch.where(shared & (old >= 0), old, NP).flatten(), torch.where((need > 0) & (new >= 0), new, NP))).long()
    refs.copy_((torch.cat((refs, refs[:1])).scatter_add_(0, more, torch.ones_like(more, dtype=I32)))[:NP])
    tails = torch.gather(old, 1, full.clamp(max=table.shape[1] - 1)[:, None].long())[:, 0]
    copies = (need > 0) & (new >= 0) & (tails >= 0)
    c_from, c_to = torch.where(copies, tails, -1), torch.where(copies, new, -1)
    c_used = torch.where(copies, used, 0)
    s["len"][dst] = ln
    # the copies, in all layers: places of the last pages that hold tokens
    at = torch.arange(p, device=DEV)[None]
    there = at < c_used[:, None]
    i, j = (c_from[:, None] * p + at)[there].long(), (c_to[:, None] * p + at)[there].long()
    for x in (s["k"], s["v"]):
        flat = x.flatten(1, 2)
        flat[:, j] = flat[:, i]
    return s["k"], s["v"], table, refs, s["len"], s["freed"], n_freed, c_from, c_to, c_used, need.sum().to(I32)[None]


# ------------------------------------------------------------------------------------------------ 64 bits

def exact(case, seed):
    if case["op"] not in ("attn", "logprobs"):
        return None                    # whole numbers and copies
    s = prepare(case, seed)
    if case["op"] == "logprobs":
        T, V = s["x"].shape
        out = {k: torch.zeros(s[k].shape, dtype=F64, device=DEV) for k in ("logprob", "lse", "entropy")}
        out["top_ids"], out["top_logprobs"] = None, torch.zeros(T, s["top"], dtype=F64, device=DEV) if s["top"] else None
        step = max(1, 40_000_000 // V)
        for a in range(0, T, step):
            y = s["x"][a:a + step].double() * s["scale"]
            z = torch.logsumexp(y, -1)
            lp = y - z[:, None]
            pr = lp.exp()
            out["lse"][a:a + step] = z
            out["entropy"][a:a + step] = -(pr * torch.where(pr > 0, lp, 0.0)).sum(-1)
            out["logprob"][a:a + step] = torch.gather(lp, 1, s["ids"][a:a + step].long())
            if s["top"]:
                out["top_logprobs"][a:a + step] = torch.topk(lp, s["top"], dim=1).values
        return out
    if work(case)["flops"] > 6e11:
        return None
    Hq, Hk, D, p, G = s["Hq"], s["Hk"], s["D"], s["page"], s["Hq"] // s["Hk"]
    T = s["q"].shape[0]
    out, lse = torch.zeros(T, Hq, D, dtype=F64, device=DEV), torch.zeros(T, Hq, dtype=F64, device=DEV)
    q = s["q"].double().view(T, Hq, D)
    rows, kvs = s["row_off"].tolist(), s["kv_len"].tolist()
    goff, pre = (s["group_off"].tolist(), s["prefix_len"].tolist()) if s["prefix_len"] is not None else ([0], [])
    for r, kv in enumerate(kvs):
        a, b = rows[r], rows[r + 1]
        n = b - a
        key, val, shared = [], [], 0
        for g in range(len(pre)):
            if goff[g] <= r < goff[g + 1]:
                shared = pre[g]
                j = torch.arange(shared, device=DEV)
                pg = s["ptable"][g].long()[j // p]
                key.append(s["k"][pg, j % p])
                val.append(s["v"][pg, j % p])
        j = torch.arange(kv, device=DEV)
        pg = s["table"][r].long()[j // p]
        key, val = torch.cat(key + [s["k"][pg, j % p]]), torch.cat(val + [s["v"][pg, j % p]])
        bits = (s["mask"][a:b, :, None].to(I64) >> torch.arange(32, device=DEV)) & 1
        sees = torch.cat((torch.ones(n, shared + kv - n, dtype=torch.bool, device=DEV), bits.flatten(1)[:, :n].bool()), 1)
        for h in range(Hk):
            sc = torch.einsum("ngd,kd->ngk", q[a:b, h * G:(h + 1) * G], key[:, h].double()) * s["scale"]
            sc.masked_fill_(~sees[:, None], -math.inf)
            z = torch.logsumexp(sc, -1)
            lse[a:b, h * G:(h + 1) * G] = z
            out[a:b, h * G:(h + 1) * G] = torch.exp(sc - z[..., None]) @ val[:, h].double()
    return out.view(T, Hq * D), lse
