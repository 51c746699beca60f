"""Attention over the paged cache, with and without shared prefixes, against the 64-bit definition.  What no row may use
holds NaN (see AttnCase), so a key too many shows."""
import numpy as np
import pytest
import torch

from serving_inputs import AttnCase

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2604_12782_b200 import binding
    return binding


def go(B, what="", max_new=0, pad=0, **kw):
    c = AttnCase(**kw)
    o, lse = c.run(B, max_new=max_new, pad=pad)
    B.osc_sync_check()
    c.check(o, lse, what or str({k: v for k, v in kw.items()})[:200])
    if pad:
        assert (c.obig[:, c.Hk * c.G * c.D:].float() == 7.0).all()
    return c


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kv", [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 200, 1000])
def test_one_token(B, D, kv):
    go(B, seed=kv, Hk=2, G=4, D=D, page=16, new=[1], kv=[kv], max_new=1)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("layout", ["nhd", "hnd", "pair"])
def test_pages_and_layouts(B, page, layout):
    go(B, seed=page, Hk=2, G=2, D=128, page=page, new=[1, 1, 1], kv=[300, 5, 77], layout=layout, pad=16)
    go(B, seed=page + 1, Hk=3, G=1, D=64, page=page, new=[2, 40, 1], kv=[300, 41, 77], prefix=[page + 9], layout=layout)
    go(B, seed=page + 2, Hk=2, G=8, D=128, page=page, new=[30, 1], kv=[300, 77], prefix=[3 * page], layout=layout, pad=8)


@pytest.mark.parametrize("G", [1, 2, 3, 4, 5, 7, 8, 12, 16, 20, 33, 64, 100, 128])
def test_group_sizes(B, G):
    go(B, seed=G, Hk=1 if G > 16 else 2, G=G, D=128 if G % 2 else 64, page=16, new=[1, 3, 1], kv=[40, 130, 9], prefix=[70])


@pytest.mark.parametrize("max_new", [0, 1, 50])
def test_ragged_steps(B, max_new):
    """The hint is a choice of kernel, the result holds whatever it says."""
    go(B, seed=1, Hk=2, G=4, D=128, page=32, new=[1, 0, 50, 1, 7, 0, 33, 1], kv=[5, 80, 50, 400, 20, 0, 200, 1], max_new=max_new, tail_rows=3)


def test_long_prompts(B):
    go(B, seed=2, Hk=1, G=4, D=128, page=64, new=[300, 129], kv=[300, 500])
    go(B, seed=3, Hk=1, G=1, D=64, page=16, new=[520], kv=[1111])
    go(B, seed=4, Hk=2, G=6, D=128, page=16, new=[65, 64, 63], kv=[65, 200, 63], prefix=[257, 128], groups=[0, 2, 3])


def test_rows_without_keys(B):
    # no own keys and no prefix; fewer own keys than new tokens; an empty prefix; requests outside every group
    go(B, seed=5, Hk=2, G=4, D=128, page=16, new=[1, 1, 3, 1], kv=[0, 4, 1, 0], tail_rows=2)
    go(B, seed=6, Hk=2, G=4, D=64, page=16, new=[1, 1, 40, 2], kv=[0, 4, 9, 1], prefix=[0, 33], groups=[0, 2, 3])
    go(B, seed=7, Hk=1, G=8, D=128, page=16, new=[0, 0], kv=[0, 0], tail_rows=4)
    go(B, seed=8, Hk=1, G=8, D=128, page=16, new=[200], kv=[3])
    go(B, seed=9, Hk=1, G=8, D=128, page=16, new=[1, 1, 1], kv=[0, 0, 0], prefix=[100], groups=[0, 2])


@pytest.mark.parametrize("R,prefix", [(1, 1), (1, 300), (4, 128), (9, 700), (33, 129), (70, 1000)])
def test_shared_prefix(B, R, prefix):
    rng = np.random.default_rng(R)
    go(B, seed=R, Hk=2, G=4, D=128, page=16, new=[1] * R, kv=list(rng.integers(0, 90, R)), prefix=[prefix], max_new=1)


def test_groups(B):
    go(B, seed=10, Hk=2, G=8, D=64, page=16, new=[1] * 12, kv=[3, 0, 40, 7, 100, 1, 1, 64, 65, 2, 0, 9], prefix=[64, 0, 300, 17],
       groups=[1, 4, 4, 9, 10])
    go(B, seed=11, Hk=1, G=2, D=128, page=32, new=[5, 1, 0, 30, 2, 2], kv=[5, 10, 12, 31, 64, 3], prefix=[90, 200, 5], groups=[0, 2, 3, 6],
       tail_rows=1)


def test_large_scores_and_one_peak(B):
    """Scores of +-100 and more: the running maximum moves, weights underflow."""
    go(B, seed=12, Hk=2, G=4, D=128, page=16, new=[1, 20], kv=[700, 300], prefix=[200], q_mul=20.0)
    c = AttnCase(13, 1, 4, 128, 16, [1], [600], q_mul=1.0)
    c.k[:] = torch.nan_to_num(c.k, nan=0.0)
    o, lse = c.run(B)
    c.check(o, lse, "finite garbage behind the end")


def test_absent_pages_read_as_zero(B):
    """A table entry outside the cache stands for keys and values of 0; nothing outside the cache is touched."""
    for new in (1, 40):
        c = AttnCase(14, 2, 4, 128, 16, [new], [100], prefix=[64])
        c.table[0, 2] = -1
        c.table[0, 4] = 2 ** 30
        c.ptable[0, 1] = c.k.shape[0]
        K, V = c.own[0]
        for lo in (32, 64):
            K[lo:lo + 16] = 0
            V[lo:lo + 16] = 0
        c.pre[0][0][16:32] = 0
        c.pre[0][1][16:32] = 0
        o, lse = c.run(B)
        B.osc_sync_check()
        c.check(o, lse, f"absent pages, {new} tokens")


def test_lengths_past_the_table_are_cut(B):
    c = AttnCase(15, 1, 4, 64, 16, [1], [48], prefix=[32])
    o1, l1 = c.run(B)
    c.kv_len.fill_(100000)
    c.prefix_len.fill_(2 ** 31 - 1)
    c.table, c.ptable = c.table[:, :3].contiguous(), c.ptable[:, :2].contiguous()
    o2, l2 = c.run(B)
    B.osc_sync_check()
    assert torch.equal(o1, o2) and torch.equal(l1, l2)


def test_unusual_offsets_stay_in_bounds(B):
    """Row offsets that fall, pass T or are negative, and groups past R: nothing outside the buffers, no fault."""
    c = AttnCase(16, 2, 4, 128, 16, [2, 2, 30], [20, 20, 40], prefix=[50])
    for rows, groups in (([0, 10, 4, 1000], [0, 3]), ([-5, 2, 2, 34], [-2, 9]), ([40, 30, 20, 10], [2, 1]), ([0, 2, 4, 34], [3, 3])):
        c.row_off.copy_(torch.tensor(rows, dtype=torch.int32))
        c.group_off.copy_(torch.tensor(groups, dtype=torch.int32))
        c.run(B)
        B.osc_sync_check()


def test_same_bits_every_time_and_without_lse(B):
    c = AttnCase(17, 2, 4, 128, 16, [1] * 20 + [70], [300 + 17 * i for i in range(20)] + [400], prefix=[900])
    o1, l1 = c.run(B)
    for _ in range(5):
        o2, l2 = c.run(B)
        assert torch.equal(o1, o2) and torch.equal(l1, l2)
    o3, _ = c.run(B, with_lse=False)
    assert torch.equal(o1, o3)


def test_streams_and_captured_step(B):
    """A captured step replayed with other lengths, two graphs on one workspace one after the other, and a side stream."""
    c = AttnCase(18, 2, 4, 128, 16, [1] * 6, [200, 5, 90, 64, 0, 33], prefix=[150], groups=[0, 6])
    d = AttnCase(19, 2, 4, 128, 16, [1] * 6, [60, 45, 199, 1, 20, 7], prefix=[150], groups=[0, 6])
    Hq, D, T = 8, 128, 6
    ws = torch.empty(B.osc_paged_attention_workspace_bytes(T, Hq, D, 6, 1), dtype=torch.uint8, device="cuda")
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    graphs = []
    with torch.cuda.stream(st):
        for x in (c, d):
            x.o = torch.full((T, Hq * D), 7.0, dtype=torch.bfloat16, device="cuda")
            x.lse = torch.full((T, Hq), 7.0, device="cuda")
            cache = B.KvCache(x.k, x.v)
            args = (x.q, cache, x.row_off, x.kv_len, x.table, x.o, ws, x.scale, x.lse, x.group_off, x.prefix_len, x.ptable, 1)
            B.osc_paged_attention(*args)
            st.synchronize()
            x.check(x.o, x.lse, "side stream")
            x.o.fill_(7.0)
            g = torch.cuda.CUDAGraph()
            st.synchronize()
            with torch.cuda.graph(g, stream=st):
                B.osc_paged_attention(*args)
            graphs.append(g)
        for _ in range(3):
            for g in graphs:
                g.replay()
        st.synchronize()
        c.check(c.o, c.lse, "graph 1")
        d.check(d.o, d.lse, "graph 2")
        kv = [100, 5, 30, 64, 0, 1]                    # shorter than the pages hold: the keys are the first ones
        c.kv_len.copy_(torch.tensor(kv, dtype=torch.int32))
        c.prefix_len.fill_(70)
        graphs[0].replay()
        st.synchronize()
    c.kv, c.prefix = kv, [70]
    c.own = [(K[:n], V[:n]) for (K, V), n in zip(c.own, kv)]
    c.pre = [(K[:70], V[:70]) for K, V in c.pre]
    c.check(c.o, c.lse, "graph 1 with other lengths")


@pytest.mark.parametrize("seed", range(12))
def test_random_steps(B, seed):
    rng = np.random.default_rng(100 + seed)
    R = int(rng.integers(1, 12))
    new = [int(rng.integers(0, 3)) if rng.random() < 0.7 else int(rng.integers(0, 90)) for _ in range(R)]
    kv = [n + int(rng.integers(0, 400)) if rng.random() < 0.8 else int(rng.integers(0, n + 1)) for n in new]
    P = int(rng.integers(0, 3))
    cuts = sorted(int(x) for x in rng.integers(0, R + 1, P + 1)) if P else None
    go(B, seed=seed, Hk=int(rng.integers(1, 4)), G=int(rng.choice([1, 2, 4, 5, 8])), D=int(rng.choice([64, 128])), page=int(rng.choice([16, 32, 64])),
       new=new, kv=kv, prefix=[int(x) for x in rng.integers(0, 500, P)], groups=cuts, tail_rows=int(rng.integers(0, 3)),
       max_new=int(rng.choice([0, 1, max(new + [1])])), pad=8 * int(rng.integers(0, 3)))


def test_offsets_past_32_bits(B):
    """A cache whose last pages lie more than 2^32 elements behind its first."""
    n_pages, page, Hk, D = 2_200_000, 16, 1, 128
    if torch.cuda.mem_get_info()[0] < 24e9:
        pytest.skip("needs 24 GB")
    c = AttnCase(20, Hk, 4, D, page, [1, 40], [500, 300], prefix=[333])
    for name in ("k", "v"):
        small = getattr(c, name)
        big = torch.empty((n_pages, page, Hk, D), dtype=torch.bfloat16, device="cuda")
        big[-small.shape[0]:] = small
        setattr(c, name, big)
    shift = n_pages - small.shape[0]
    for t in (c.table, c.ptable):
        t.copy_(torch.where((t >= 0) & (t < small.shape[0]), t + shift, t))
        t.copy_(torch.where(t < n_pages, t, n_pages + 5))
    o, lse = c.run(B)
    B.osc_sync_check()
    c.check(o, lse, "far pages")


def test_many_units_to_a_share(B):
    """Prompts long enough that every CTA of the kernel for many rows runs through several units, with lists that end inside tiles
    of all kinds, one after the other."""
    go(B, seed=21, Hk=8, G=4, D=128, page=64, new=[700, 3, 650, 900], kv=[1000, 900, 650, 1111], prefix=[391])
    go(B, seed=22, Hk=8, G=8, D=64, page=16, new=[500, 333, 420], kv=[777, 640, 421], prefix=[129, 70], groups=[0, 2, 3])


@pytest.mark.parametrize("R,P,G", [(257, 0, 4), (300, 3, 4), (1100, 2, 2), (1300, 0, 1), (700, 600, 1)])
def test_many_requests(B, R, P, G):
    """More requests and groups than the plan handles in one go."""
    rng = np.random.default_rng(R)
    new = list(rng.choice([0, 1, 2], R, p=[0.1, 0.8, 0.1]))
    kv = [int(n + rng.integers(0, 40)) for n in new]
    go(B, seed=R, Hk=1, G=G, D=64, page=16, new=new, kv=kv, prefix=[int(x) for x in rng.integers(0, 60, P)], tail_rows=1)


@pytest.mark.parametrize("D", [64, 128])
def test_long_and_short_requests_of_one_group(B, D):
    """Prompts and single tokens behind the same prefix; a second group of prompts only."""
    go(B, seed=21, Hk=2, G=4, D=D, page=16, new=[70, 1, 300, 0, 33, 1], kv=[90, 40, 300, 7, 500, 0], prefix=[200])
    go(B, seed=22, Hk=1, G=8, D=D, page=32, new=[100, 1, 64, 40, 130], kv=[100, 300, 64, 300, 131], prefix=[333, 90], groups=[0, 2, 5], tail_rows=2)


def test_tokens_in_front_of_the_first_request(B):
    """Rows in front of row_off[0] are left as they were, whatever the workspace held."""
    for fill in (0, 1, 0x7F):
        c = AttnCase(23, 2, 4, 128, 16, [1, 1, 40, 1], [30, 4, 60, 9], prefix=[100, 50], groups=[0, 2, 4])
        front, Hq, D = 5, 8, 128
        q = torch.full((c.T + front, Hq * D), float("nan"), dtype=torch.bfloat16, device="cuda")
        q[front:] = c.q
        o = torch.full_like(q, 7.0)
        lse = torch.full((c.T + front, Hq), 7.0, device="cuda")
        ws = torch.full((B.osc_paged_attention_workspace_bytes(c.T + front, Hq, D, 4, 2) // 4,), fill, dtype=torch.int32, device="cuda")
        ws = ws.view(torch.uint8)
        B.osc_paged_attention(q, B.KvCache(c.k, c.v), c.row_off + front, c.kv_len, c.table, o, ws, c.scale, lse=lse, group_off=c.group_off,
                              prefix_len=c.prefix_len, prefix_table=c.ptable)
        B.osc_sync_check()
        c.check(o[front:], lse[front:], f"front rows, workspace of {fill}")
        assert (o[:front].float() == 7.0).all() and (lse[:front] == 7.0).all()


def test_no_requests_and_no_tokens(B):
    c = AttnCase(24, 2, 4, 64, 16, [0, 0], [5, 0], prefix=[20])
    o, lse = c.run(B)
    B.osc_sync_check()
    c.check(o, lse, "no tokens")
    d = AttnCase(25, 2, 4, 64, 16, [1], [5], tail_rows=2)
    o, lse = torch.full((3, 512), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((3, 8), 7.0, device="cuda")
    ws = torch.zeros(B.osc_paged_attention_workspace_bytes(3, 8, 64, 0, 0), dtype=torch.uint8, device="cuda")
    B.osc_paged_attention(d.q, B.KvCache(d.k, d.v), d.row_off[:1], d.kv_len[:0], d.table[:0], o, ws, d.scale, lse=lse)
    B.osc_sync_check()
    assert (o.float() == 7.0).all() and (lse == 7.0).all()


def test_two_streams_at_once(B):
    """Two steps under way at once, each with its own workspace."""
    cases = [AttnCase(26, 2, 4, 128, 16, [1] * 40 + [90], [700] * 41, prefix=[1500]), AttnCase(27, 4, 8, 128, 16, [1] * 9, [5000] * 9)]
    streams, bufs = [torch.cuda.Stream() for _ in cases], []
    for c in cases:
        Hq, R, P = c.Hk * c.G, len(c.new), len(c.prefix)
        bufs.append((torch.full((c.T, Hq * c.D), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((c.T, Hq), 7.0, device="cuda"),
                     torch.zeros(B.osc_paged_attention_workspace_bytes(c.T, Hq, c.D, R, P), dtype=torch.uint8, device="cuda")))
    torch.cuda.synchronize()
    for _ in range(8):
        for c, (o, lse, ws), st in zip(cases, bufs, streams):
            P = len(c.prefix)
            B.osc_paged_attention(c.q, B.KvCache(c.k, c.v), c.row_off, c.kv_len, c.table, o, ws, c.scale, lse=lse, group_off=c.group_off,
                                  prefix_len=c.prefix_len, prefix_table=c.ptable if P else None, stream=st)
    torch.cuda.synchronize()
    for c, (o, lse, _) in zip(cases, bufs):
        c.check(o, lse, "two streams")


@pytest.mark.parametrize("kv", [50, 300, 700])
def test_many_units(B, kv):
    """More row units in one request than the line is laid out for in a loop: some without keys, some short, some behind a prefix."""
    go(B, seed=28, Hk=1, G=64, D=64, page=16, new=[300, 1], kv=[kv, 40])
    go(B, seed=29, Hk=1, G=128, D=64, page=16, new=[150, 150], kv=[kv, 160], prefix=[130])
    go(B, seed=30, Hk=2, G=8, D=64, page=16, new=[200, 3], kv=[kv, 40], max_new=1)


def test_a_cache_without_pages(B):
    """Every table entry is outside the cache: keys and values of 0, so a row that sees any key gives 0 and ln(number of keys)."""
    for new, kv, P in (([1, 1], [5, 70], 0), ([1, 40], [5, 70], 1), ([3], [0], 0)):
        T, R, Hq, D = sum(new), len(new), 8, 128
        q = torch.randn(T, Hq * D, device="cuda").to(torch.bfloat16)
        k = torch.empty(0, 16, 2, D, dtype=torch.bfloat16, device="cuda")
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")     # noqa: E731
        o, lse = torch.full((T, Hq * D), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((T, Hq), 7.0, device="cuda")
        ws = torch.zeros(B.osc_paged_attention_workspace_bytes(T, Hq, D, R, P), dtype=torch.uint8, device="cuda")
        rows = np.concatenate([[0], np.cumsum(new)])
        B.osc_paged_attention(q, B.KvCache(k, k.clone()), i32(rows.tolist()), i32(kv), torch.zeros(R, 8, dtype=torch.int32, device="cuda"), o, ws, 0.1, lse=lse,
                              group_off=i32([0, R]) if P else None, prefix_len=i32([30]) if P else None,
                              prefix_table=torch.zeros(1, 2, dtype=torch.int32, device="cuda") if P else None)
        B.osc_sync_check()
        assert (o == 0).all()
        sees = np.concatenate([np.maximum(m - n + np.arange(n) + 1, 0) for n, m in zip(new, kv)]) + 30 * P
        with np.errstate(divide="ignore"):
            want = np.log(sees)
        got = lse.cpu().numpy().astype(np.float64)
        # ex2, lg2 and the sums are off by a few 2^-22 of ln(n) + 1
        assert (np.abs(np.where(sees[:, None] > 0, got - np.where(sees > 0, want, 0)[:, None], 0)) <= 2.0 ** -18 * 6).all()
        assert (got[sees == 0] == -np.inf).all()


@pytest.mark.parametrize("page", [512, 4096])
def test_large_pages_and_tables_with_a_stride(B, page):
    c = AttnCase(31, 2, 4, 128, page, [1, 60, 1], [700, 1300, 9], prefix=[600, 20], groups=[0, 2, 3])
    wide = torch.full((3, c.table.shape[1] + 5), 2 ** 31 - 1, dtype=torch.int32, device="cuda")
    wide[:, :c.table.shape[1]] = c.table
    c.table = wide[:, :c.table.shape[1]]
    pwide = torch.full((2, c.ptable.shape[1] + 3), -2 ** 31, dtype=torch.int32, device="cuda")
    pwide[:, :c.ptable.shape[1]] = c.ptable
    c.ptable = pwide[:, :c.ptable.shape[1]]
    o, lse = c.run(B)
    B.osc_sync_check()
    c.check(o, lse, f"pages of {page}")


@pytest.mark.parametrize("max_new", [0, 1])
def test_falling_offsets_compute_nothing(B, max_new):
    """Requests or groups that would share rows: no row is written (with and without prefixes, so by either way of planning)."""
    c = AttnCase(32, 4, 4, 128, 16, [2, 2, 30], [20, 20, 40], prefix=[50])
    for rows, groups in (([0, 10, 4, 34], [0, 3]), ([0, 34, 0, 34], [0, 3]), ([40, 30, 20, 10], [0, 3]), ([0, 2, 4, 34], [3, 0])):
        c.row_off.copy_(torch.tensor(rows, dtype=torch.int32))
        c.group_off.copy_(torch.tensor(groups, dtype=torch.int32))
        o, lse = c.run(B, max_new=max_new)
        B.osc_sync_check()
        assert (o.float() == 7.0).all() and (lse == 7.0).all()
    d = AttnCase(33, 4, 4, 128, 16, [2, 2, 30], [20, 20, 1])
    for rows in ([0, 10, 4, 34], [0, 34, 0, 34], [40, 30, 20, 10]):
        d.row_off.copy_(torch.tensor(rows, dtype=torch.int32))
        o, lse = d.run(B, max_new=max_new)
        B.osc_sync_check()
        assert (o.float() == 7.0).all() and (lse == 7.0).all()


def same_bits(a, b):
    return torch.equal(a.contiguous().view(torch.int16), b.contiguous().view(torch.int16))


NAN_STEPS = {
    # name: (case, maximum of new tokens, tokens of which one head's query is NaN)
    "whole units, few rows": (dict(seed=34, Hk=4, G=4, D=128, page=16, new=[1, 1, 1], kv=[16, 9, 3]), 1, [1]),
    "cut units, few rows": (dict(seed=35, Hk=4, G=4, D=128, page=16, new=[1, 1], kv=[600, 700]), 1, [0]),
    "cut units, few rows, joined warps": (dict(seed=36, Hk=1, G=4, D=64, page=16, new=[1, 1], kv=[3000, 2500]), 1, [0]),
    "whole units, many rows": (dict(seed=37, Hk=2, G=4, D=128, page=16, new=[60, 64], kv=[100, 64]), 0, [3, 70]),
    "cut units, many rows": (dict(seed=38, Hk=1, G=4, D=128, page=64, new=[20, 70], kv=[2500, 4000]), 0, [5, 40]),
    "cut units of 64 channels": (dict(seed=39, Hk=1, G=8, D=64, page=16, new=[9, 40], kv=[2500, 4000]), 0, [5, 30]),
    "behind a prefix, few rows": (dict(seed=40, Hk=2, G=4, D=128, page=16, new=[1, 1, 1], kv=[300, 5, 0], prefix=[700]), 1, [0, 2]),
    "behind a prefix, many rows": (dict(seed=41, Hk=2, G=4, D=128, page=16, new=[1] * 30 + [30], kv=[40] * 31, prefix=[900]), 0, [4, 45]),
    "a prompt behind a prefix": (dict(seed=42, Hk=1, G=4, D=128, page=16, new=[130], kv=[500], prefix=[3000]), 0, [100]),
}


@pytest.mark.parametrize("name", NAN_STEPS)
def test_a_nan_query_gives_nan_and_leaves_its_neighbours(B, name):
    """However its keys are cut, a head whose query is NaN gives NaN, not the 0 and -inf of a row without keys."""
    kw, max_new, tokens = NAN_STEPS[name]
    c = AttnCase(**kw)
    Hq, D = c.Hk * c.G, c.D
    o, lse = c.run(B, max_new=max_new)
    c.check(o, lse, name)
    clean, clean_lse = o.clone(), lse.clone()
    hit = torch.zeros(c.T, Hq, dtype=torch.bool, device="cuda")
    for i, t in enumerate(tokens):
        h = (5 * i + 2) % Hq
        hit[t, h] = True
        c.q[t, h * D:(h + 1) * D] = float("nan")
    o, lse = c.run(B, max_new=max_new)
    B.osc_sync_check()
    o, clean = o.reshape(c.T, Hq, D), clean.reshape(c.T, Hq, D)
    assert torch.isnan(o[hit].float()).all() and torch.isnan(lse[hit]).all(), f"{name}: NaN was lost"
    o[hit], lse[hit] = clean[hit], clean_lse[hit]
    c.check(o.reshape(c.T, Hq * D), lse, f"{name}, neighbours")      # (rows of one tile are rescaled together, so not bit for bit)


@pytest.mark.parametrize("new,max_new", [(1, 1), (40, 0)])
@pytest.mark.parametrize("kv", [60, 3000])
@pytest.mark.parametrize("prefix", [[], [500]])
def test_a_nan_key_gives_nan_where_it_is_seen(B, new, max_new, kv, prefix):
    """One key of one request holds NaN: every row of that request and head gives NaN, in whichever piece the key lies, and nobody else."""
    for at in (0, kv // 2, kv - new):
        c = AttnCase(43, 2, 4, 128, 16, [1, new, 1], [70, kv, 20], prefix=prefix)
        Hq, D = 8, 128
        o, lse = c.run(B, max_new=max_new)
        clean, clean_lse = o.clone().reshape(c.T, Hq, D), lse.clone()
        c.k[int(c.table[1, at // 16]), at % 16, 1, 3] = float("nan")
        o, lse = c.run(B, max_new=max_new)
        B.osc_sync_check()
        o = o.reshape(c.T, Hq, D)
        hit = torch.zeros(c.T, Hq, dtype=torch.bool, device="cuda")
        hit[1 + max(at - (kv - new), 0):1 + new, 4:] = True          # token i of the request sees own keys up to kv - new + i
        assert torch.isnan(o[hit].float()).all() and torch.isnan(lse[hit]).all(), f"key {at}"
        assert same_bits(o[~hit], clean[~hit]) and torch.equal(lse[~hit], clean_lse[~hit]), f"key {at}"


def test_rows_of_o_in_the_gaps_of_q(B):
    """Q and O as columns of one buffer, and a single token right behind another: the same as in buffers of their own."""
    for kw, max_new in ((dict(seed=44, Hk=2, G=4, D=128, page=16, new=[1, 40, 1], kv=[300, 77, 9], prefix=[90]), 0),
                        (dict(seed=45, Hk=4, G=2, D=64, page=16, new=[1], kv=[500]), 1)):
        c = AttnCase(**kw)
        o, lse = c.run(B, max_new=max_new)
        w, P = c.Hk * c.G * c.D, len(c.prefix)
        buf = torch.full((c.T, 2 * w), 7.0, dtype=torch.bfloat16, device="cuda")
        buf[:, :w] = c.q
        ws = torch.zeros(B.osc_paged_attention_workspace_bytes(c.T, c.Hk * c.G, c.D, len(c.new), P), dtype=torch.uint8, device="cuda")
        lse2 = torch.full_like(lse, 7.0)
        B.osc_paged_attention(buf[:, :w], B.KvCache(c.k, c.v), c.row_off, c.kv_len, c.table, buf[:, w:], ws, c.scale, lse=lse2,
                              group_off=c.group_off, prefix_len=c.prefix_len, prefix_table=c.ptable if P else None, max_new=max_new)
        B.osc_sync_check()
        assert same_bits(buf[:, w:], o) and torch.equal(lse, lse2) and same_bits(buf[:, :w], c.q)


class Guarded:
    """A buffer with 64 KB of marked bytes on either side."""
    EDGE = 1 << 16

    def __init__(self, nbytes, fill):
        self.all = torch.full((nbytes + 2 * self.EDGE + 512,), 0xA5, dtype=torch.uint8, device="cuda")
        self.nbytes = nbytes
        self.all[self.EDGE:self.EDGE + nbytes] = fill

    def view(self, dtype, *shape):
        return self.all[self.EDGE:self.EDGE + self.nbytes].view(dtype).view(*shape)

    def intact(self):
        return bool((self.all[:self.EDGE] == 0xA5).all() and (self.all[self.EDGE + self.nbytes:] == 0xA5).all())


@pytest.mark.parametrize("max_new", [0, 1])
@pytest.mark.parametrize("rows,groups,new,group_rows", [
    ([0, 10, 4, 1000], [0, 3], None, None), ([40, 30, 20, 10], [2, 1], None, None), ([0, 2, 4, 34], [3, 0], None, None),
    ([-5, 2, 2, 34], [-2, 9], [2, 0, 32], [0, 3]), ([0, 2, 4, 34], [3, 3], [2, 2, 30], [3, 3]), ([-7, -1, 6, 99], [1, 40], [0, 6, 28], [1, 3])])
def test_unusual_offsets_inside_marked_buffers(B, max_new, rows, groups, new, group_rows):
    """Offsets outside [0, T] count as cut to it; where they fall no row is written.  Nothing around O, lse and the workspace changes."""
    c = AttnCase(16, 2, 4, 128, 16, [2, 2, 30], [20, 20, 40], prefix=[50])
    T, Hq, D = c.T, 8, 128
    need = B.osc_paged_attention_workspace_bytes(T, Hq, D, 3, 1)
    go_, gl, gw = Guarded(T * Hq * D * 2, 0), Guarded(T * Hq * 4, 0), Guarded(need, 0xFF)
    o, lse = go_.view(torch.bfloat16, T, Hq * D), gl.view(torch.float32, T, Hq)
    o.fill_(7.0)
    lse.fill_(7.0)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")      # noqa: E731
    B.osc_paged_attention(c.q, B.KvCache(c.k, c.v), i32(rows), c.kv_len, c.table, o, gw.view(torch.uint8, need), c.scale, lse=lse,
                          group_off=i32(groups), prefix_len=c.prefix_len, prefix_table=c.ptable, max_new=max_new)
    B.osc_sync_check()
    assert go_.intact() and gl.intact() and gw.intact(), "written outside the buffers"
    if new is None:
        assert (o == 7.0).all() and (lse == 7.0).all()
        return
    c.new, c.groups, c.rows = new, group_rows, np.concatenate([[0], np.cumsum(new)]).astype(int)
    c.check(o, lse, f"rows {rows}, groups {groups}")


@pytest.mark.parametrize("new,max_new", [([1, 1, 1], 1), ([3, 40, 1], 0)])
def test_tables_without_columns(B, new, max_new):
    """Requests that hold no key of their own: the prefix alone, or nothing."""
    for prefix, groups in (([70], [0, 2]), ([], None)):
        c = AttnCase(46, 2, 4, 128, 16, new, [0, 0, 0], prefix=prefix, groups=groups)
        c.table = torch.empty(3, 0, dtype=torch.int32, device="cuda")
        o, lse = c.run(B, max_new=max_new)
        B.osc_sync_check()
        c.check(o, lse, f"prefix {prefix}")


def test_calls_of_all_kinds_share_a_workspace_one_behind_the_other(B):
    """Layers and steps of a model back to back on one stream, by every way of planning, with one workspace between them: the same bits as with
    the device idle between calls."""
    kinds = [(dict(Hk=4, G=4, D=128, page=16, new=[1] * 7, kv=[900, 3, 40, 2000, 1, 77, 600]), 1),
             (dict(Hk=2, G=4, D=128, page=16, new=[1] * 30 + [70], kv=[300 + 7 * i for i in range(31)], prefix=[1500]), 0),
             (dict(Hk=2, G=8, D=64, page=32, new=[1] * 12, kv=[50 * i for i in range(12)], prefix=[700, 90], groups=[0, 5, 11]), 1),
             (dict(Hk=8, G=4, D=128, page=64, new=[400, 1, 300], kv=[700, 900, 300]), 0),
             (dict(Hk=1, G=16, D=64, page=16, new=[1] * 3, kv=[4000, 10, 0]), 1),
             (dict(Hk=2, G=4, D=128, page=16, new=[260, 300], kv=[500, 300], prefix=[333]), 0)]
    cases = [(AttnCase(50 + i, **kw), max_new) for i, (kw, max_new) in enumerate(kinds * 2)]
    ws = torch.empty(max(B.osc_paged_attention_workspace_bytes(c.T, c.Hk * c.G, c.D, len(c.new), len(c.prefix)) for c, _ in cases),
                     dtype=torch.uint8, device="cuda")
    caches = [B.KvCache(c.k, c.v) for c, _ in cases]

    def outputs():
        return [(torch.full((c.T, c.Hk * c.G * c.D), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((c.T, c.Hk * c.G), 7.0, device="cuda"))
                for c, _ in cases]

    def call(i, out):
        c, max_new = cases[i]
        B.osc_paged_attention(c.q, caches[i], c.row_off, c.kv_len, c.table, out[i][0], ws, c.scale, lse=out[i][1], group_off=c.group_off,
                              prefix_len=c.prefix_len, prefix_table=c.ptable if c.prefix else None, max_new=max_new)
    alone = outputs()
    for i, (c, _) in enumerate(cases):
        ws.fill_(0xFF)
        call(i, alone)
        B.osc_sync_check()
        if i < len(kinds):
            c.check(*alone[i], f"kind {i}")
    rng = np.random.default_rng(0)
    for _ in range(20):
        out = outputs()
        torch.cuda.synchronize()
        for i in rng.permutation(len(cases)):
            call(int(i), out)
        B.osc_sync_check()
        for i, ((o, lse), (ro, rl)) in enumerate(zip(out, alone)):
            assert same_bits(o, ro) and torch.equal(lse, rl), f"call {i}"
