"""Moves in the paged cache: accepted tokens, pages given back, forks and copies.  Whole numbers and copies: equal to the plain definitions."""
import numpy as np
import pytest
import torch

from oracle import branching

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2604_12782_b200 import binding
    return binding


def dev(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def host(t):
    return t.cpu().numpy()


def layers_of(B, L, n_pages, page, Hk, D, seed, layout="nhd"):
    """(handle, list of the layers' K and V as [n_pages, page, Hk, D] views): distinct values everywhere, NaN bit patterns among them."""
    g = torch.Generator(device="cuda").manual_seed(seed)

    def bits(*shape):
        return torch.randint(-2 ** 15, 2 ** 15, shape, generator=g, device="cuda", dtype=torch.int16).view(torch.bfloat16)
    out = []
    for _ in range(L):
        if layout == "nhd":
            out.append((bits(n_pages, page, Hk, D), bits(n_pages, page, Hk, D)))
        elif layout == "hnd":
            out.append(tuple(bits(n_pages, Hk, page, D).permute(0, 2, 1, 3) for _ in range(2)))
        else:                              # keys and values side by side, rows further apart than they are long
            both = bits(n_pages, page, 2, Hk, D + 8)
            out.append((both[:, :, 0, :, :D], both[:, :, 1, :, :D]))
    return B.KvLayers([B.KvCache(k, v) for k, v in out]), out


def raw(t):
    return t.contiguous().view(torch.int16).cpu().numpy()


class Compact:
    def __init__(self, B, seed, L, Hk, D, page, new, ctx, keep, keep_cols=None, layout="nhd", ld_pad=0):
        rng = np.random.default_rng(seed)
        R = len(new)
        kv = np.array(new) + np.array(ctx)
        counts = [-(-int(x) // page) for x in kv]
        n_pages = sum(counts) + 2
        order = list(rng.permutation(n_pages))
        self.tab = np.full((R, max(counts + [0]) + 1), n_pages + 3, np.int64)
        for r, c in enumerate(counts):
            for j in range(c):
                self.tab[r, j] = order.pop()
        cols = keep_cols if keep_cols is not None else max([len(k) for k in keep] + [0])
        self.n_keep = np.array([len(k) for k in keep])
        self.keep = np.full((R, cols), 123456, np.int64)
        for r, k in enumerate(keep):
            self.keep[r, :min(len(k), cols)] = k[:cols]
        self.rows, self.kv, self.ld_pad = np.concatenate([[0], np.cumsum(new)]), kv, ld_pad
        self.layers, self.kvs = layers_of(B, L, n_pages, page, Hk, D, seed, layout)

    def check(self, B):
        before = [(raw(k), raw(v)) for k, v in self.kvs]
        R = len(self.kv)
        big = torch.full((R, self.keep.shape[1] + self.ld_pad), 5, dtype=torch.int32, device="cuda")
        big[:, :self.keep.shape[1]] = dev(self.keep)
        new_len = torch.full((R + 1,), 77, dtype=torch.int32, device="cuda")
        B.osc_kv_compact(self.layers, dev(self.rows), dev(self.kv), dev(self.tab), big[:, :self.keep.shape[1]], dev(self.n_keep), new_len)
        for (k, v), b in zip(self.kvs, before):
            for t, x in zip((k, v), b):
                want, length = branching.kv_compact(x, self.rows, self.kv, self.tab, self.keep, self.n_keep)
                assert np.array_equal(raw(t), want)
        assert np.array_equal(host(new_len), np.append(length, 77))


@pytest.mark.parametrize("L,Hk,D,page,layout", [(1, 8, 128, 16, "nhd"), (3, 4, 64, 64, "hnd"), (2, 1, 64, 1, "side"), (36, 8, 128, 128, "nhd"), (5, 3, 128, 5, "side"),
                                                (130, 1, 64, 16, "nhd")])
def test_compact(B, L, Hk, D, page, layout):
    rng = np.random.default_rng(L)
    new = [26, 1, 64, 0, 7, 40]
    keep = [sorted(rng.choice(n, rng.integers(0, n + 1), replace=False)) for n in new]
    Compact(B, L, L, Hk, D, page, new, [100, 0, 31, 8, 16, 3], keep, layout=layout, ld_pad=L % 3).check(B)


def test_compact_all_none_and_many(B):
    Compact(B, 1, 2, 2, 64, 16, [10, 10, 10], [5, 5, 5], [list(range(10)), [], [9]]).check(B)
    rng = np.random.default_rng(2)
    new = rng.integers(0, 9, 700)
    Compact(B, 2, 2, 1, 64, 16, new, rng.integers(0, 40, 700), [sorted(rng.choice(n, rng.integers(0, n + 1), replace=False)) for n in new]).check(B)


def test_compact_long_lists(B):
    """More entries than one round takes, every move onto a place that another entry has just left."""
    rng = np.random.default_rng(3)
    Compact(B, 3, 2, 2, 64, 16, [1500, 900], [70, 3], [list(range(1, 1500)), sorted(rng.choice(900, 600, replace=False))]).check(B)
    Compact(B, 4, 1, 8, 128, 64, [300], [10], [list(range(44, 300))]).check(B)


@pytest.mark.parametrize("keep", [[3, 3, 4], [5, 2, 6], [0, 1, 26], [-1, 4], [0, 2, 2 ** 31 - 1], [26], [4, -2 ** 31], [1, 3, 5, 4]])
def test_lists_end_where_indices_do_not_rise(B, keep):
    Compact(B, 5, 2, 2, 64, 16, [26, 30], [20, 7], [keep, [1, 29]]).check(B)


def test_compact_odd_arguments(B):
    c = Compact(B, 6, 1, 2, 64, 16, [9, 12, 5], [20, 7, 40], [[2, 4], [1, 5, 8], [0, 3]])
    c.n_keep = np.array([5, -3, 2])               # more than the columns, less than none
    c.check(B)
    c = Compact(B, 7, 1, 2, 64, 16, [9, 12], [20, 40], [[2, 4, 8], [1, 5, 8]])
    c.tab[0, 1], c.tab[1, 3] = -1, 10 ** 9        # pages that are not there
    c.check(B)
    c = Compact(B, 8, 1, 2, 64, 16, [9, 12], [20, 40], [[2, 4, 8], [1, 5, 8]])
    c.kv = np.array([4, 2 ** 31 - 1])             # fewer tokens than new ones; past the table
    c.check(B)
    c = Compact(B, 9, 2, 2, 64, 16, [4], [5], [[1, 3]], keep_cols=0)
    c.check(B)
    c = Compact(B, 10, 2, 2, 64, 16, [3, 4], [5, 6], [[1, 2], [3]])
    c.rows = np.array([0, 3, 1])                  # falling offsets: no new tokens
    c.check(B)


class Trim:
    def __init__(self, seed, lens, to, page, cols=None, shared=0, refs=True, spare=3, ld_pad=0):
        rng = np.random.default_rng(seed)
        R = len(lens)
        counts = [-(-max(int(x), 0) // page) for x in lens]
        cols = max(counts + [0]) + 1 if cols is None else cols
        self.n_pages = sum(min(c, cols) for c in counts) + spare
        order = list(rng.permutation(self.n_pages))
        self.tab = np.full((R, cols), -1, np.int64)
        for r, c in enumerate(counts):
            for j in range(min(c, cols)):
                self.tab[r, j] = order.pop()
        if shared:                           # rows behind the first hold its first pages too
            for r in range(1, R):
                n = min(shared, counts[0], counts[r], cols)
                self.tab[r, :n] = self.tab[0, :n]
        self.refs = np.bincount(self.tab[self.tab >= 0], minlength=self.n_pages) if refs else None
        self.lens, self.to, self.page, self.ld_pad = lens, to, page, ld_pad

    def check(self, B):
        R, cols = self.tab.shape
        big = torch.full((R, cols + self.ld_pad), 77, dtype=torch.int32, device="cuda")
        big[:, :cols] = dev(self.tab)
        refs = dev(self.refs) if self.refs is not None else None
        freed, n_freed = torch.full((self.n_pages + 2,), 77, dtype=torch.int32, device="cuda"), dev([5, 5])
        B.osc_kv_trim(dev(self.lens), dev(self.to), self.page, big[:, :cols], refs, freed, n_freed, n_pages=self.n_pages)
        tab, want, gone = branching.kv_trim(self.lens, self.to, self.page, self.tab, self.refs, self.n_pages)
        assert n_freed.tolist() == [len(gone), 5]
        assert np.array_equal(host(freed), np.concatenate([gone, np.full(self.n_pages + 2 - len(gone), 77)]))
        assert np.array_equal(host(big[:, :cols]), tab) and (big[:, cols:] == 77).all()
        if refs is not None:
            assert np.array_equal(host(refs), want)
        # nothing is left to give back
        B.osc_kv_trim(dev(self.lens), dev(self.to), self.page, big[:, :cols], refs, freed, n_freed, n_pages=self.n_pages)
        assert n_freed.tolist() == [0, 5] and np.array_equal(host(big[:, :cols]), tab)


@pytest.mark.parametrize("R,page,most", [(1, 16, 100), (7, 64, 5000), (513, 16, 300), (1100, 1, 40), (3, 128, 100000)])
@pytest.mark.parametrize("refs", [True, False])
def test_trim(B, R, page, most, refs):
    rng = np.random.default_rng(R)
    lens = rng.integers(0, most, R)
    to = np.where(rng.random(R) < 0.4, 0, np.where(rng.random(R) < 0.5, lens, rng.integers(0, most, R)))
    Trim(R, lens, to, page, refs=refs, ld_pad=R % 3).check(B)


def test_trim_shared_pages(B):
    """A page is freed with its last holder, once, whatever the order."""
    Trim(1, [200] * 40, [0] * 40, 16, shared=9).check(B)
    Trim(2, [200] * 40, [0] * 39 + [200], 16, shared=9).check(B)
    Trim(3, [500, 77, 130, 500], [300, 0, 130, 17], 16, shared=31).check(B)


def test_trim_odd_arguments(B):
    t = Trim(4, [100, 60], [0, 0], 16)
    t.refs = np.where(np.arange(t.n_pages) % 3 == 0, 0, t.refs)       # counts that say nobody holds the page
    t.refs[1] = -4
    t.check(B)
    t = Trim(5, [100, 60, -5], [-7, 200, 3], 16)
    t.check(B)
    t = Trim(6, [2 ** 31 - 1, 60], [10, 0], 16, cols=5)               # lengths past the table's columns
    t.check(B)
    t = Trim(7, [100, 60], [0, 0], 16)
    t.tab[0, 1], t.tab[1, 2], t.tab[1, 0] = 10 ** 9, -5, t.n_pages
    t.check(B)
    t = Trim(8, [100, 60], [0, 0], 16, shared=3)                      # more holders than the count says
    t.refs[:] = 1
    t.check(B)


def test_trim_without_requests_or_columns(B):
    n_freed, freed = dev([9]), dev([4, 4, 4])
    empty = torch.zeros(0, dtype=torch.int32, device="cuda")
    B.osc_kv_trim(empty, empty, 16, torch.zeros(0, 4, dtype=torch.int32, device="cuda"), None, freed, n_freed)
    assert n_freed.item() == 0 and freed.tolist() == [4, 4, 4]
    B.osc_kv_trim(dev([50, 3]), dev([0, 0]), 16, torch.zeros(2, 0, dtype=torch.int32, device="cuda"), None, freed, n_freed)
    assert n_freed.item() == 0


def test_trim_many_pages(B):
    """A bitmap of a million pages, freed from all over it."""
    rng = np.random.default_rng(9)
    n_pages, R, cols = 1_000_003, 64, 500
    tab = rng.choice(n_pages, R * cols, replace=False).reshape(R, cols)
    tab[0, :3] = [0, n_pages - 1, 31]
    lens, to = np.full(R, cols * 16), np.where(np.arange(R) % 3 == 1, 100, 0)
    table, freed, n_freed = dev(tab), torch.full((n_pages,), -7, dtype=torch.int32, device="cuda"), dev([0])
    B.osc_kv_trim(dev(lens), dev(to), 16, table, None, freed, n_freed)
    want, _, gone = branching.kv_trim(lens, to, 16, tab, None, n_pages)
    assert n_freed.item() == len(gone) and np.array_equal(host(freed[:len(gone)]), gone) and (freed[len(gone):] == -7).all()
    assert np.array_equal(host(table), want)


class Fork:
    def __init__(self, seed, R, n, page, most, refs=True, n_free=None, cols=None, ld_pad=0):
        rng = np.random.default_rng(seed)
        rows = rng.permutation(R)
        self.dst, live = rows[:n], rows[n:]
        self.src = rng.choice(live, n)
        self.len = rng.integers(0, most, R)
        self.len[live[0]] = most // page * page
        counts = -(-self.len // page)
        cols = int(counts.max()) + 1 if cols is None else cols
        n_free = n + 3 if n_free is None else n_free
        self.n_pages = int(counts.sum()) + n_free + 4
        order = rng.permutation(self.n_pages)
        self.tab = np.full((R, cols), -1, np.int64)
        at = 0
        for r in range(R):
            m = min(int(counts[r]), cols)
            self.tab[r, :m] = order[at:at + m]
            at += m
        self.free = order[at:at + n_free]
        self.refs = np.bincount(self.tab[self.tab >= 0], minlength=self.n_pages) if refs else None
        self.page, self.ld_pad = page, ld_pad

    def check(self, B):
        R, cols = self.tab.shape
        n = len(self.src)
        big = torch.full((R, cols + self.ld_pad), 77, dtype=torch.int32, device="cuda")
        big[:, :cols] = dev(self.tab)
        refs, length = dev(self.refs) if self.refs is not None else None, dev(self.len)
        c = [torch.full((n + 1,), 77, dtype=torch.int32, device="cuda") for _ in range(3)]
        taken = dev([5, 5])
        B.osc_kv_fork(dev(self.src), dev(self.dst), length, self.page, dev(self.free), big[:, :cols], refs, *c, taken, n_pages=self.n_pages)
        tab, want, ln, copies, took = branching.kv_fork(self.src, self.dst, self.len, self.page, self.free, self.tab, self.refs, self.n_pages)
        assert taken.tolist() == [took, 5]
        assert np.array_equal(host(big[:, :cols]), tab) and (big[:, cols:] == 77).all()
        assert np.array_equal(host(length), ln)
        for j in range(3):
            assert np.array_equal(host(c[j]), np.append(copies[:, j], 77))
        if refs is not None:
            assert np.array_equal(host(refs), want)


@pytest.mark.parametrize("R,n,page,most", [(2, 1, 16, 100), (4, 3, 64, 777), (300, 290, 16, 200), (1100, 700, 1, 40), (9, 4, 32, 60000), (5, 0, 16, 50)])
@pytest.mark.parametrize("refs", [True, False])
def test_fork(B, R, n, page, most, refs):
    Fork(R, R, n, page, most, refs=refs, ld_pad=R % 4).check(B)


def test_fork_odd_arguments(B):
    f = Fork(1, 12, 6, 16, 90)
    f.src[0], f.src[1], f.dst[2], f.dst[3] = -1, 12, 2 ** 31 - 1, -5
    f.src[4] = f.dst[4]
    f.check(B)
    f = Fork(2, 12, 6, 16, 90, n_free=2)                 # the free list runs out
    f.check(B)
    f = Fork(3, 12, 6, 16, 90)
    f.free[1], f.free[2] = 10 ** 9, -3                   # pages that are not there in the list
    f.check(B)
    f = Fork(4, 12, 6, 16, 200, cols=4)                  # lengths past the table's columns
    f.check(B)
    f = Fork(5, 12, 6, 16, 90)
    f.tab[f.src[0], 0] = f.n_pages
    f.tab[f.src[1], 1] = -9
    f.len[f.src[2]] = -4
    f.check(B)


@pytest.mark.parametrize("L,Hk,D,page,n,layout", [(1, 8, 128, 16, 1, "nhd"), (36, 8, 128, 32, 7, "nhd"), (3, 4, 64, 64, 40, "hnd"), (2, 3, 128, 5, 9, "side"),
                                                  (130, 1, 64, 16, 2, "nhd"), (1, 8, 128, 1024, 1, "hnd"), (2, 1, 64, 1, 30, "side")])
@pytest.mark.parametrize("whole", [False, True])
def test_copy_pages(B, L, Hk, D, page, n, layout, whole):
    rng = np.random.default_rng(n)
    n_pages = 2 * n + 3
    order = rng.permutation(n_pages)
    a, b = order[:n].copy(), order[n:2 * n].copy()
    used = rng.integers(0, page + 1, n)
    if n > 6:
        a[1], b[2], a[3], used[4], used[5] = -1, n_pages, 2 ** 31 - 1, -2, 10 ** 6
        b[6] = a[6]
        a[5] = a[0]                                      # one page copied twice
    layers, kvs = layers_of(B, L, n_pages, page, Hk, D, n, layout)
    before = [(raw(k), raw(v)) for k, v in kvs]
    B.osc_kv_copy_pages(layers, dev(a), dev(b), None if whole else dev(used))
    for (k, v), x in zip(kvs, before):
        for t, want in zip((k, v), x):
            want = want.copy()
            for i in range(n):
                if 0 <= a[i] < n_pages and 0 <= b[i] < n_pages and a[i] != b[i]:
                    m = page if whole else min(max(int(used[i]), 0), page)
                    want[b[i], :m] = want[a[i], :m]
            assert np.array_equal(raw(t), want)


def test_gaps_between_rows_keep_their_bytes(B):
    both = torch.full((6, 16, 2, 2, 72), 7.0, dtype=torch.bfloat16, device="cuda")
    both[..., :64] = torch.randn(6, 16, 2, 2, 64, device="cuda")
    k, v = both[:, :, 0, :, :64], both[:, :, 1, :, :64]
    layers = B.KvLayers([B.KvCache(k, v)])
    B.osc_kv_copy_pages(layers, dev([0, 1]), dev([2, 3]), dev([16, 9]))
    B.osc_kv_compact(layers, dev([0, 9]), dev([20]), dev([[4, 5]]), dev([[1, 3, 8]]), dev([3]), dev([0]))
    assert (both[..., 64:] == 7).all()


def test_captured_and_on_another_stream(B):
    """A step of a beam search, captured once and replayed on other contents."""
    layers, kvs = layers_of(B, 3, 40, 16, 2, 64, 1)
    table, refs = torch.full((6, 8), -1, dtype=torch.int32, device="cuda"), torch.zeros(40, dtype=torch.int32, device="cuda")
    length, to, src, dst, free = dev([0] * 6), dev([0] * 6), dev([0, 0]), dev([0, 0]), dev([0] * 8)
    freed, n_freed, taken, c = torch.full((40,), -1, dtype=torch.int32, device="cuda"), dev([0]), dev([0]), [dev([0, 0]) for _ in range(3)]

    def step():
        B.osc_kv_trim(length, to, 16, table, refs, freed, n_freed)
        B.osc_kv_fork(src, dst, length, 16, free, table, refs, *c, taken)
        B.osc_kv_copy_pages(layers, *c)
    s = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        step()
    for seed in (1, 2, 3):
        rng = np.random.default_rng(seed)
        n = rng.integers(1, 60, 6)
        order = rng.permutation(40)
        tab, at = np.full((6, 8), -1, np.int64), 0
        for r in range(6):
            m = -(-int(n[r]) // 16)
            tab[r, :m] = order[at:at + m]
            at += m
        hold = np.bincount(tab[tab >= 0], minlength=40)
        fr = np.concatenate([order[at:], np.full(8, -1)])[:8]
        a, b = np.array([1, 4]), np.array([0, 5])
        sh = np.where(np.isin(np.arange(6), b), 0, n)
        for t, x in ((table, tab), (refs, hold), (length, n), (to, sh), (src, a), (dst, b), (free, fr)):
            t.copy_(dev(x))
        before = [(raw(k), raw(v)) for k, v in kvs]
        g.replay()
        torch.cuda.synchronize()
        t1, h1, gone = branching.kv_trim(n, sh, 16, tab, hold, 40)
        t2, h2, l2, copies, took = branching.kv_fork(a, b, n, 16, fr, t1, h1, 40)
        assert np.array_equal(host(table), t2) and np.array_equal(host(refs), h2) and np.array_equal(host(length), l2)
        assert n_freed.item() == len(gone) and np.array_equal(host(freed)[:len(gone)], gone) and taken.item() == took
        for (k, v), x in zip(kvs, before):
            for t, want in zip((k, v), x):
                want = want.copy()
                for p, q, m in copies:
                    if p >= 0:
                        want[q, :m] = want[p, :m]
                assert np.array_equal(raw(t), want)


def test_a_cache_past_31_bits_of_elements(B):
    """Pages whose offsets pass 2^31 elements."""
    page, Hk, D = 16, 8, 128
    big = torch.empty(3 * 45000, page, Hk, D, dtype=torch.bfloat16, device="cuda")      # 2.2e9 elements
    kk, vv = big[0::3], big[1::3]
    n = kk.shape[0]
    for p in (0, 1, n - 1, n - 2):
        kk[p].copy_(torch.randn(page, Hk, D, device="cuda"))
        vv[p].copy_(torch.randn(page, Hk, D, device="cuda"))
    layers = B.KvLayers([B.KvCache(kk, vv)])
    B.osc_kv_copy_pages(layers, dev([0, n - 1]), dev([n - 3, 5]))
    assert torch.equal(kk[n - 3], kk[0]) and torch.equal(vv[5], vv[n - 1])
    want = [t[n - 1, 5].clone() for t in (kk, vv)]
    B.osc_kv_compact(layers, dev([0, 8]), dev([24]), dev([[n - 2, n - 1]]), dev([[0, 5]]), dev([2]), dev([0]))
    # context 16 tokens on page n - 2, new tokens on page n - 1: new token 5 moves to place 1
    assert torch.equal(kk[n - 1, 1], want[0]) and torch.equal(vv[n - 1, 1], want[1])


def test_layers_next_to_one_another(B):
    """Keys and values that alternate through one buffer, handed over in another order than they lie in: no two layers share any."""
    n, L = 6, 40
    both = torch.arange(n * 16 * 2 * L * 64, device="cuda", dtype=torch.int32).to(torch.int16).view(torch.bfloat16).view(n, 16, 2 * L, 1, 64)
    order = np.random.default_rng(5).permutation(2 * L)
    caches = [B.KvCache(both[:, :, int(order[2 * i])], both[:, :, int(order[2 * i + 1])]) for i in range(L)]
    want = branching.kv_compact(raw(both), [0, 9], [20], np.array([[4, 5]]), np.array([[1, 3, 8]]), [3])[0]
    B.osc_kv_compact(B.KvLayers(caches), dev([0, 9]), dev([20]), dev([[4, 5]]), dev([[1, 3, 8]]), dev([3]), dev([0]))
    assert np.array_equal(raw(both), want)
    with pytest.raises(B.OscError, match="another layer"):
        B.osc_kv_compact(B.KvLayers(caches + caches[:1]), dev([0, 9]), dev([20]), dev([[4, 5]]), dev([[1, 3, 8]]), dev([3]), dev([0]))
    assert np.array_equal(raw(both), want)
