"""Pages, slots and positions from request lengths: whole numbers, equal to the plain definition."""
import numpy as np
import pytest
import torch

from oracle import serving

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2604_12782_b200 import binding
    return binding


def dev(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


class Step:
    def __init__(self, seed, cached, fresh, page, T=None, n_free=None, cols=None, with_base=True, ld_pad=0):
        rng = np.random.default_rng(seed)
        R = len(cached)
        c, n = np.maximum(cached, 0), np.maximum(fresh, 0)
        held = -(-c // page)
        need = int((-(-(c + n) // page) - held).sum())
        cols = int(max(-(-(c + n) // page)) if R else 0) + 1 if cols is None else cols
        n_free = need + 3 if n_free is None else n_free
        pages = rng.permutation(int(held.sum()) + n_free + 10)
        self.table = np.full((R, cols), -9, np.int64)
        at = 0
        for r in range(R):
            m = min(int(held[r]), cols)
            self.table[r, :m] = pages[at:at + m]
            at += m
        self.free = pages[at:at + n_free]
        self.cached, self.fresh, self.page = cached, fresh, page
        self.base = rng.integers(0, 100000, R) if with_base else None
        self.T = int(n.sum()) if T is None else T
        self.ld_pad = ld_pad

    def run(self, B, stream=None):
        R, cols = self.table.shape
        big = torch.full((R, cols + self.ld_pad), 77, dtype=torch.int32, device="cuda")
        big[:, :cols] = dev(self.table.reshape(R, cols))
        tab = big[:, :cols]
        out = dict(row_off=dev(np.full(R + 2, 5)), kv_len=dev(np.full(R + 1, 5)), slots=dev(np.full(self.T, 5)), positions=dev(np.full(self.T, 5)),
                   taken=dev([5, 5]))
        B.osc_kv_slots(dev(self.cached), dev(self.fresh), dev(self.base) if self.base is not None else None, self.page, dev(self.free), tab,
                       out["row_off"], out["kv_len"], out["slots"], out["positions"], out["taken"], stream=stream)
        return big, tab, out

    def check(self, B):
        big, tab, out = self.run(B)
        torch.cuda.synchronize()
        R, cols = self.table.shape
        row, kv, table, slots, pos, taken = serving.kv_slots(self.cached, self.fresh, self.base, self.page, self.free, self.table, self.T)
        assert np.array_equal(out["row_off"].cpu().numpy(), np.append(row, 5))
        assert np.array_equal(out["kv_len"].cpu().numpy(), np.append(kv, 5))
        assert out["taken"].tolist() == [taken, 5]
        assert np.array_equal(tab.cpu().numpy(), table)
        assert np.array_equal(out["slots"].cpu().numpy(), slots)
        assert np.array_equal(out["positions"].cpu().numpy(), pos)
        assert (big[:, cols:] == 77).all()


@pytest.mark.parametrize("R,page", [(1, 16), (2, 1), (31, 16), (511, 32), (512, 16), (513, 64), (1500, 7), (2100, 128)])
def test_decoding_step(B, R, page):
    rng = np.random.default_rng(R)
    Step(R, rng.integers(0, 700, R), np.ones(R, int), page).check(B)


@pytest.mark.parametrize("R,page,most", [(1, 16, 5000), (3, 64, 3000), (40, 16, 900), (600, 32, 60), (1100, 5, 30)])
def test_prompts_and_empty_requests(B, R, page, most):
    rng = np.random.default_rng(R + 1)
    fresh = rng.integers(0, most, R)
    fresh[rng.random(R) < 0.3] = 0
    cached = rng.integers(0, 300, R)
    cached[rng.random(R) < 0.3] = 0
    Step(R, cached, fresh, page, ld_pad=3).check(B)


def test_lengths_at_page_ends(B):
    cached = np.array([0, 0, 0, 15, 15, 16, 16, 17, 31, 32, 0])
    fresh = np.array([15, 16, 17, 1, 2, 0, 1, 15, 1, 0, 0])
    Step(0, cached, fresh, 16, with_base=False).check(B)


def test_filled_up_step_short_list_narrow_table_negative_lengths(B):
    rng = np.random.default_rng(9)
    cached, fresh = rng.integers(0, 100, 50), rng.integers(0, 40, 50)
    Step(1, cached, fresh, 16, T=int(fresh.sum()) + 1000).check(B)        # rows behind the tokens: slot -1, position 0
    Step(2, cached, fresh, 16, T=int(fresh.sum()) - 100).check(B)         # fewer rows than tokens
    Step(3, cached, fresh, 16, n_free=20).check(B)                        # the list runs out
    Step(4, cached, fresh, 16, n_free=0).check(B)
    Step(5, cached, fresh, 16, cols=4).check(B)                           # requests wider than the table
    fresh[::7] = -5
    cached[::5] = -1
    Step(6, cached, fresh, 16).check(B)
    Step(7, np.zeros(0, int), np.zeros(0, int), 16, T=10).check(B)
    Step(8, np.zeros(4, int), np.zeros(4, int), 16, T=0).check(B)


def test_far_positions_and_same_outputs_twice(B):
    s = Step(11, np.array([2_000_000, 5]), np.array([700, 3]), 128)
    s.check(B)
    big, tab, out = s.run(B)
    first = [tab.clone()] + [v.clone() for v in out.values()]
    B.osc_kv_slots(dev(s.cached), dev(s.fresh), dev(s.base), s.page, dev(s.free), tab, out["row_off"], out["kv_len"], out["slots"],
                   out["positions"], out["taken"])
    assert all(torch.equal(a, b) for a, b in zip(first, [tab] + list(out.values())))


def test_captured_step_follows_the_lengths(B):
    s = Step(12, np.array([3, 40, 0]), np.array([1, 1, 5]), 16, T=64)
    R, cols = s.table.shape[0], 20
    table = dev(np.concatenate([s.table, np.full((R, cols - s.table.shape[1]), -9)], 1))
    cached, fresh, free = dev(s.cached), dev(s.fresh), dev(np.arange(100, 200))
    out = [dev(np.zeros(n)) for n in (R + 1, R, 64, 64, 1)]
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(st):
        B.osc_kv_slots(cached, fresh, None, 16, free, table, *out)
        st.synchronize()
        with torch.cuda.graph(g, stream=st):
            B.osc_kv_slots(cached, fresh, None, 16, free, table, *out)
    for c, n in (([3, 40, 0], [1, 1, 5]), ([4, 41, 5], [2, 7, 20]), ([0, 0, 0], [0, 64, 0])):
        cached.copy_(dev(c))
        fresh.copy_(dev(n))
        before = table.cpu().numpy()
        g.replay()
        torch.cuda.synchronize()
        row, kv, tab, slots, pos, taken = serving.kv_slots(c, n, None, 16, np.arange(100, 200), before, 64)
        for got, want in zip(out + [table], (row, kv, slots, pos, [taken], tab)):
            assert np.array_equal(got.cpu().numpy(), np.asarray(want))


@pytest.mark.parametrize("page", [1 << 16, 1 << 20])
def test_lengths_whose_sum_passes_32_bits(B, page):
    """However long the requests behind them are, the first T tokens get their slots; counts stop at 2^31 - 1."""
    big = 2 ** 31 - 1
    for seed, cached, fresh in ((20, [5, 0, 0, 7], [3, big, big, 4]), (21, [0, 9], [big, 2]), (22, [100, 0, 0, 0], [2, 2 ** 30, 2 ** 30, 2 ** 30]),
                                (23, [0] * 2, [big] * 2), (24, [3] + [0] * 700, [5] + [big] * 700), (25, [0] * 300 + [4], [1] * 300 + [big])):
        s = Step(seed, np.array(cached), np.array(fresh), page, T=400, n_free=600, cols=40)
        s_tab = s.table.copy()
        _, tab, out = s.run(B)
        torch.cuda.synchronize()
        c, n = np.array(cached, np.int64), np.array(fresh, np.int64)
        rows, grown = np.concatenate([[0], np.cumsum(n)]), -(-(c + n) // page) - -(-c // page)
        first = np.concatenate([[0], np.cumsum(grown)])
        assert np.array_equal(out["row_off"].cpu().numpy()[:len(c) + 1], np.minimum(rows, big))
        assert np.array_equal(out["kv_len"].cpu().numpy()[:len(c)], np.minimum(c + n, big))
        assert out["taken"].tolist()[0] == min(int(first[-1]), big)
        for r in range(len(c)):
            for j in range(int(grown[r])):
                col, f = -(-int(c[r]) // page) + j, int(first[r]) + j
                if col >= 40:
                    break
                s_tab[r, col] = s.free[f] if f < 600 else -1
        assert np.array_equal(tab.cpu().numpy(), s_tab)
        slots, pos = np.full(400, -1, np.int64), np.zeros(400, np.int64)
        for t in range(min(400, int(rows[-1]))):
            r = int(np.searchsorted(rows, t, side="right")) - 1
            at = int(c[r]) + t - int(rows[r])
            p = int(s_tab[r, at // page]) if at // page < 40 else -1
            slots[t], pos[t] = (p * page + at % page if p >= 0 and p * page + at % page < 2 ** 31 else -1), s.base[r] + at
        assert np.array_equal(out["slots"].cpu().numpy(), slots) and np.array_equal(out["positions"].cpu().numpy(), pos)


def test_tokens_at_the_end_of_the_range(B):
    """A request whose cached tokens end within a page of 2^31."""
    page, cols = 1 << 20, 2048
    table = torch.arange(cols, dtype=torch.int32, device="cuda")[None].flip(1).contiguous()
    for cached, fresh in ((2 ** 31 - 9, 4), (2 ** 31 - page - 3, 6), (2 ** 31 - page, 2)):
        tab, T = table.clone(), 8
        held = -(-cached // page)
        tab[0, held:] = -9
        out = [dev(np.full(n, 5)) for n in (2, 1, T, T, 1)]
        B.osc_kv_slots(dev([cached]), dev([fresh]), None, page, dev([17, 18]), tab, *out)
        torch.cuda.synchronize()
        row, kv, tab_ref, slots, pos, taken = serving.kv_slots([cached], [fresh], None, page, [17, 18], np.where(np.arange(cols) < held, 2047 - np.arange(cols), -9)[None], T)
        assert (slots[:fresh] < 2 ** 31).all()
        for got, want in zip(out + [tab], (row, kv, slots, pos, [taken], tab_ref)):
            assert np.array_equal(got.cpu().numpy(), np.asarray(want))
