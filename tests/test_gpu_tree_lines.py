"""Masked attention where a step has work for both kernels, and where the tcgen05 kernel lays out many requests by itself, against the
64-bit definition.  (Requests of up to 16 rows a key/value head may go to the few-row kernel, prefixes and larger trees to the tcgen05 kernel; where
requests have more rows than that on average, all go to the latter.)"""
import numpy as np
import pytest
import torch

from branching_inputs import TreeCase

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2604_12782_b200 import binding
    return binding


def on_both(c):
    """Whether the step has a request for either kernel, and the mean that leaves them there."""
    few = [n for n in c.new if 0 < n * c.G <= 16]
    return few and sum(c.new) * c.G <= len(c.new) * 16 and (c.prefix or max(c.new) * c.G > 16)


# key/value heads: units of four, two and one head on the few-row line
@pytest.mark.parametrize("Hk,G,D", [(4, 4, 128), (2, 4, 128), (1, 4, 64), (3, 2, 128), (8, 4, 64)])
@pytest.mark.parametrize("prefix,kv", [(300, 60), (4100, 200), (90, 900)])
def test_small_drafts_behind_a_prefix(B, Hk, G, D, prefix, kv):
    """The prefix on the tcgen05 line, own keys with the mask on the few-row line, every row with two sources."""
    rng = np.random.default_rng(prefix + Hk)
    new = [int(x) for x in rng.integers(1, 5, 12)]
    own = [n + int(rng.integers(0, kv)) for n in new]
    for style in ("tree", "any"):
        c = TreeCase(5, Hk, G, D, 16, new, own, prefix=[prefix], style=style, tail_rows=3)
        assert on_both(c)
        c.check(*c.run(B, max_new=4), what=style)
        c.check(*c.run(B), what=style + ", most new tokens not given")


@pytest.mark.parametrize("Hk,G,D", [(4, 4, 128), (2, 4, 128), (1, 4, 64), (3, 2, 128)])
@pytest.mark.parametrize("kv", [30, 700, 3000])
def test_a_tree_among_single_tokens(B, Hk, G, D, kv):
    """One tree on the tcgen05 line, twenty requests of one or two tokens on the few-row line; both lines cut into shares inside units."""
    rng = np.random.default_rng(kv + Hk)
    new = [int(x) for x in rng.integers(1, 3, 20)]
    new.insert(7, 26)
    own = [n + int(rng.integers(kv // 2, kv)) for n in new]
    c = TreeCase(6, Hk, G, D, 16, new, own, tail_rows=2)
    assert on_both(c)
    c.check(*c.run(B, max_new=26))


def test_groups_of_both_kinds(B):
    """A group of small drafts, one whose requests fill row tiles (their prefix and own keys are one list), requests in no group."""
    new = [2, 3, 1, 4, 70, 66, 1, 2, 3] + [1] * 45
    kv = [50, 3, 200, 90, 400, 66, 800, 2, 60] + [40 + i for i in range(45)]
    for Hk, G, D in ((4, 4, 128), (2, 2, 64)):
        c = TreeCase(9, Hk, G, D, 32, new, kv, prefix=[700, 1300], groups=[0, 4, 6])
        assert on_both(c)
        c.check(*c.run(B, max_new=70))


def test_contexts_cut_on_both_lines(B):
    c = TreeCase(13, 4, 4, 128, 64, [3, 40, 2, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1], [9000, 12000, 7000, 5000] + [60] * 10)
    assert on_both(c)
    c.check(*c.run(B, max_new=40))


def test_odd_values_on_both_lines(B):
    new, kv = [3, 40] + [1] * 20, [90, 3000] + [300] * 20
    c = TreeCase(14, 4, 4, 128, 16, new, kv, style="any")
    assert on_both(c)
    for r, m in ((0, 1), (1, 39), (1, 0), (5, 0)):
        c.spoil(r, m, [0, 127], float("nan"))
        c.spoil(r, m, [64], float("inf"))
    c.check_odd(*c.run(B, max_new=40))


# up to 256 requests without prefixes the tcgen05 kernel lays out its line for itself, a thread to a request; 257: the plan kernel does
@pytest.mark.parametrize("R,Hk,G,D", [(R, 1, 8, 64) for R in (2, 31, 32, 33, 64, 255, 256, 257, 300)] + [(R, 2, 8, 128) for R in (2, 33, 256, 257)])
def test_many_requests(B, R, Hk, G, D):
    """Empty requests, requests without keys, fewer keys than tokens; units of one and of two row tiles in turn."""
    rng = np.random.default_rng(R)
    new = [int(rng.choice([0, 1, 5, 12, 20, 33, 40])) for _ in range(R)]
    new[0], new[-1] = 20, 33
    kv = [int(n + rng.integers(0, 200)) if rng.random() < 0.8 else int(rng.integers(0, max(n, 1))) if rng.random() < 0.5 else 0 for n in new]
    kv[-1] = 133
    assert sum(new) * G > R * 16
    c = TreeCase(R, Hk, G, D, 16, new, kv, tail_rows=R % 3)
    c.check(*c.run(B, max_new=40))


@pytest.mark.parametrize("new,kv,prefix", [([26], [926], []), ([40] * 6, [4000] * 6, []), ([3] * 12, [300] * 12, [4100]), ([1] * 20 + [26], [900] * 21, [])])
def test_calls_repeat_themselves(B, new, kv, prefix):
    """The same call on the same inputs gives the same bits, whatever ran between: pieces are joined in the order of the keys."""
    c = TreeCase(17, 4, 4, 128, 16, new, kv, prefix=prefix)
    o, lse = c.run(B)
    junk = torch.empty(1 << 25, device="cuda")
    for i in range(6):
        if i % 2:
            junk.normal_()
        o2, lse2 = c.run(B)
        assert torch.equal(o.view(torch.int16), o2.view(torch.int16)) and torch.equal(lse.view(torch.int32), lse2.view(torch.int32)), i


@pytest.mark.parametrize("new,kv", [([3, 20], 96), ([2, 1, 1], 64)])
def test_lengths_past_the_table_are_cut(B, new, kv):
    """To what the columns hold, the new tokens being the last keys of that."""
    c = TreeCase(15, 4, 4, 128, 16, new, [kv] * len(new), prefix=[32])
    o, lse = c.run(B)
    c.kv_len.fill_(100000)
    c.prefix_len.fill_(2 ** 31 - 1)
    c.table, c.ptable = c.table[:, :kv // 16].contiguous(), c.ptable[:, :2].contiguous()
    o2, lse2 = c.run(B)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
