"""Trees of drafted tokens: masks and positions equal to the plain definition, attention against the 64-bit definition."""
import numpy as np
import pytest
import torch

from branching_inputs import TreeCase, random_parents
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


def check_mask(B, parents, new, words, tail=0, base=True, ld_pad=0, seed=0, positions=True):
    rng = np.random.default_rng(seed)
    rows = np.concatenate([[0], np.cumsum(new)]).astype(int)
    T = int(rows[-1]) + tail
    parents = np.concatenate([parents, rng.integers(-3, 9, tail)])
    base = rng.integers(0, 10 ** 6, len(new)) if base else None
    big = torch.full((T, words + ld_pad), 77, dtype=torch.int32, device="cuda")
    pos = torch.full((T + 1,), 77, dtype=torch.int32, device="cuda") if positions else None
    B.osc_tree_mask(dev(parents), dev(rows), dev(base) if base is not None else None, big[:, :words], pos)
    bits, want = branching.tree_mask(parents, rows, base, words)
    assert np.array_equal(big[:, :words].cpu().numpy(), branching.packed(bits))
    assert (big[:, words:] == 77).all()
    if positions:
        assert np.array_equal(pos.cpu().numpy(), np.append(want, 77))


@pytest.mark.parametrize("n,words", [(1, 1), (2, 1), (31, 1), (32, 1), (33, 2), (64, 2), (65, 4), (200, 7), (1024, 32), (1000, 32), (70, 1), (300, 3)])
def test_mask_of_one_request(B, n, words):
    check_mask(B, random_parents(np.random.default_rng(n), n), [n], words, tail=n % 3, seed=n)


@pytest.mark.parametrize("R,most,words", [(3, 5, 1), (50, 40, 2), (2500, 12, 1), (700, 90, 3)])
def test_masks_of_many_requests(B, R, most, words):
    rng = np.random.default_rng(R)
    new = rng.integers(0, most, R)
    check_mask(B, np.concatenate([random_parents(rng, n) for n in new] + [np.zeros(0, int)]), new, words, tail=11, ld_pad=R % 4, seed=R)


@pytest.mark.parametrize("parents", [[-1, -2, 0, 1, 2, 5, 3], [0, -1, 1, 1], [5, 4, 3, 2, 1, 0], [-7, 0, 1, 2, -1, 4], [-1] * 40, [-1] + list(range(39)),
                                     [-1, 2 ** 31 - 1, -2 ** 31, 1, 0]])
def test_tokens_that_are_not_there(B, parents):
    """Parents outside the request, at or behind the token itself: the token is not there, nor are its descendants."""
    check_mask(B, parents, [len(parents)], 2)
    check_mask(B, parents * 3, [len(parents)] * 3, 1, base=False)


def test_mask_without_positions_and_without_requests(B):
    check_mask(B, random_parents(np.random.default_rng(1), 20), [20], 1, positions=False)
    check_mask(B, [], [], 3, tail=300, base=False)
    check_mask(B, [], [0, 0, 0], 2, tail=5)


FORMS = [
    # Hk, G, D, page, new, kv: up to 16 rows a head, up to 128, up to 256, several units, and mixtures
    (8, 4, 128, 16, [4], [900]),
    (8, 4, 128, 16, [26], [926]),
    (8, 4, 128, 64, [60], [700]),
    (8, 4, 128, 64, [129], [129]),
    (4, 8, 128, 16, [1, 2, 3, 17, 33], [5, 2, 700, 17, 300]),
    (2, 7, 128, 32, [12, 1, 40], [500, 90, 41]),
    (1, 5, 64, 16, [3, 26], [77, 4000]),
    (4, 1, 64, 128, [64, 2, 5], [1000, 64, 5]),
    (8, 2, 64, 16, [8, 8, 9], [8, 130, 257]),
    (2, 16, 128, 16, [1, 9, 16], [200, 9, 128 + 16]),
    (1, 128, 128, 32, [3, 1], [100, 40]),
    (3, 4, 128, 16, [5, 31], [64, 63]),
    (6, 2, 64, 64, [2, 70], [640, 127]),
]


@pytest.mark.parametrize("form", FORMS, ids=[f"{f[0]}x{f[1]}x{f[2]}-{len(f[4])}" for f in FORMS])
@pytest.mark.parametrize("style", ["tree", "any"])
def test_attention(B, form, style):
    c = TreeCase(7, *form, style=style, tail_rows=2)
    c.check(*c.run(B), what=str(form))


@pytest.mark.parametrize("form", FORMS[:6], ids=[str(i) for i in range(6)])
def test_most_new_tokens_is_a_choice_of_kernel(B, form):
    """The result holds whatever max_new says, also where it is wrong."""
    c = TreeCase(8, *form)
    for m in (1, max(form[4]), 1000):
        c.check(*c.run(B, max_new=m), what=f"max_new {m}")


@pytest.mark.parametrize("kv", [26, 27, 64, 127, 128, 129, 150, 154, 155, 256, 282, 513])
@pytest.mark.parametrize("G,D", [(4, 128), (2, 64)])
def test_trees_across_the_edges_of_key_tiles(B, kv, G, D):
    c = TreeCase(kv, 4, G, D, 16, [26], [kv])
    c.check(*c.run(B, max_new=26), what=f"{kv} keys")


@pytest.mark.parametrize("kv", [3, 15, 16, 17, 31, 48, 50, 66])
@pytest.mark.parametrize("Hk", [4, 2, 1])
def test_few_rows_across_the_edges_of_key_tiles(B, kv, Hk):
    c = TreeCase(kv, Hk, 4, 128, 16, [3, 3], [kv, kv + 1])
    c.check(*c.run(B, max_new=3), what=f"{kv} keys")


@pytest.mark.parametrize("prefix,groups,new,kv", [
    ([40], None, [3, 26, 1], [3, 100, 70]),
    ([300, 17], None, [4, 30, 60, 2], [4, 30, 90, 500]),
    ([129], [1, 3], [5, 40, 2, 33], [60, 40, 2, 40]),
    ([0, 200], None, [9, 9], [9, 20]),
    ([500], None, [70, 80], [70, 300]),               # every request fills row tiles: prefix and own keys are one list
    ([130, 64], [0, 2, 4], [64, 100, 64, 3], [64, 200, 65, 3]),
])
def test_behind_shared_prefixes(B, prefix, groups, new, kv):
    for D, G in ((128, 4), (64, 2)):
        c = TreeCase(11, 4, G, D, 16, new, kv, prefix=prefix, groups=groups, tail_rows=1)
        c.check(*c.run(B), what=str((D, G)))


@pytest.mark.parametrize("form", [(8, 4, 128, 16, [5, 3], [5, 3]), (4, 4, 128, 16, [40, 2], [40, 2]), (4, 2, 64, 32, [70], [60]), (8, 4, 128, 16, [4, 3], [2, 0]),
                                  (4, 8, 128, 64, [33, 1, 2], [0, 0, 1])])
def test_rows_that_see_nothing(B, form):
    """No bits and no context, no keys at all, fewer keys than new tokens: 0 and -inf, whatever the values hold."""
    c = TreeCase(3, *form, style="none", tail_rows=1)
    o, lse = c.run(B)
    c.check(o, lse)
    n = int(c.rows[-1])
    for r, (x, kv) in enumerate(zip(c.new, c.kv)):
        if kv <= x:
            assert (o[c.rows[r]:c.rows[r] + x] == 0).all() and (lse[c.rows[r]:c.rows[r] + x] == -float("inf")).all()
    assert (o[n:] == 7).all()
    c = TreeCase(4, *form, style="any")
    c.check(*c.run(B))


@pytest.mark.parametrize("Hk,G,D,new,kv", [(4, 4, 128, [4, 3], [40, 90]), (4, 4, 128, [26], [300]), (2, 4, 64, [60, 40], [200, 40]), (1, 4, 128, [3], [19]),
                                           (8, 2, 64, [8, 8], [8, 140]), (4, 8, 128, [30], [2000])])
def test_odd_values_reach_only_rows_that_see_them(B, Hk, G, D, new, kv):
    """NaN and Inf among the values of new tokens: padding that no row sees, tokens that some rows see."""
    for style in ("tree", "any"):
        c = TreeCase(21, Hk, G, D, 16, new, kv, style=style)
        for r, n in enumerate(new):
            if kv[r] < n:
                continue
            c.spoil(r, n - 1, [0, D - 1], float("nan"))
            c.spoil(r, 0, [1, D // 2], float("inf"))
            c.spoil(r, n // 2, [3], -float("inf"))
            c.spoil(r, 1, [D // 2 + 1], float("nan"))
        c.check_odd(*c.run(B), what=style)


def test_odd_values_in_split_requests(B):
    """A long context is cut into pieces: the piece that holds the new tokens adds what is odd."""
    for new in ([4], [33]):
        c = TreeCase(22, 4, 4, 128, 64, new, [9000])
        c.spoil(0, 1, [5], float("nan"))
        c.spoil(0, 2, [6, 127], float("inf"))
        c.check_odd(*c.run(B, max_new=new[0]))


def test_odd_keys_of_tokens_that_are_not_seen(B):
    c = TreeCase(23, 4, 4, 128, 16, [5, 40], [50, 90], style="tree")
    for r, m in ((0, 4), (1, 39)):
        c.bits[:, m] = False
        at = c.kv[r] - c.new[r] + m
        c.k[int(c.table[r, at // 16]), at % 16] = float("nan")
        c.v[int(c.table[r, at // 16]), at % 16] = float("nan")
    c.mask = torch.from_numpy(branching.packed(c.bits)).cuda()
    c.check(*c.run(B))


@pytest.mark.parametrize("words,new", [(1, [40, 33]), (2, [70]), (1, [100, 2])])
def test_more_new_tokens_than_bits(B, words, new):
    """New tokens without a bit are seen by nobody; their rows see by their own bits."""
    c = TreeCase(31, 4, 4, 128, 16, new, [n + 50 for n in new], words=words, style="any", ld_pad=3)
    c.check(*c.run(B))


@pytest.mark.parametrize("layout", ["hnd", "side"])
def test_layouts_and_strides(B, layout):
    c = TreeCase(41, 4, 4, 128, 32, [3, 50], [70, 200], layout=layout, ld_pad=5)
    c.check(*c.run(B, pad=8))
    assert (c.obig[:, 4 * 4 * 128:] == 7).all()


def test_a_chain_equals_paged_attention(B):
    """Trees that are chains are prompts: the same keys for every row, so the outputs agree within the order of the sums."""
    new, kv = [5, 40, 200], [300, 41, 260]
    c = TreeCase(51, 8, 4, 128, 16, new, kv)
    c.bits[:] = np.concatenate([np.tril(np.ones((n, 32 * c.words), bool)) for n in new])
    c.mask = torch.from_numpy(branching.packed(c.bits)).cuda()
    o, lse = c.run(B)
    c.check(o, lse)
    from serving_inputs import AttnCase
    AttnCase.check(c, *AttnCase.run(c, B))


def test_long_contexts_split_over_the_machine(B):
    c = TreeCase(61, 4, 4, 128, 64, [20, 3], [12000, 7000])
    c.check(*c.run(B, max_new=20))


def test_another_stream_and_a_captured_graph(B):
    c = TreeCase(71, 8, 4, 128, 16, [26, 2], [300, 90])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        o, lse = c.run(B)
    s.synchronize()
    c.check(o, lse)
    # replays follow the buffers: other lengths, another mask
    Hq, D = 32, 128
    d = TreeCase(72, 8, 4, 128, 16, [20, 8], [290, 60])
    q, o, lse = c.q.clone(), torch.zeros(28, Hq * D, dtype=torch.bfloat16, device="cuda"), torch.zeros(28, Hq, device="cuda")
    row, kv, tab, mask = c.row_off.clone(), c.kv_len.clone(), torch.full((2, 24), -1, dtype=torch.int32, device="cuda"), c.mask.clone()
    ws = torch.empty(B.osc_paged_attention_workspace_bytes(28, Hq, D, 2), dtype=torch.uint8, device="cuda")
    k, v = torch.empty(60, 16, 8, D, dtype=torch.bfloat16, device="cuda"), torch.empty(60, 16, 8, D, dtype=torch.bfloat16, device="cuda")

    def fill(x):
        q.copy_(x.q)
        row.copy_(x.row_off)
        kv.copy_(x.kv_len)
        tab[:, :x.table.shape[1]] = x.table
        mask.copy_(x.mask)
        k[:x.k.shape[0]] = x.k
        v[:x.v.shape[0]] = x.v
    fill(c)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.osc_tree_attention(q, B.KvCache(k, v), row, kv, tab, mask, o, ws, c.scale, lse=lse)
    for x in (c, d, c):
        fill(x)
        o.fill_(7)
        lse.fill_(7)
        g.replay()
        torch.cuda.synchronize()
        x.check(o, lse)


@pytest.mark.parametrize("new", [[3, 2], [40, 9]])
def test_a_cache_without_pages(B, new):
    """Every key reads as zero: equal weights, O = 0, lse = ln of the number of keys that a row sees."""
    c = TreeCase(91, 4, 4, 128, 16, new, [n + 20 for n in new])
    want = np.concatenate([np.log(c.sees(r).sum(1)) for r in range(2)])
    c.k, c.v = (torch.zeros(0, 16, 4, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    o, lse = c.run(B)
    torch.cuda.synchronize()
    assert (o == 0).all() and np.abs(lse.cpu().numpy() - want[:, None]).max() < 1e-5
    # pages that are not there, in a cache that has some
    c = TreeCase(91, 4, 4, 128, 16, new, [n + 20 for n in new])
    c.table[:] = torch.where(torch.arange(c.table.shape[1], device="cuda") % 2 == 0, -1, 10 ** 9).int()
    o, lse = c.run(B)
    torch.cuda.synchronize()
    assert (o == 0).all() and np.abs(lse.cpu().numpy() - want[:, None]).max() < 1e-5


def test_offsets_that_fall_write_no_row_twice(B):
    """Contents are the caller's; whatever they hold nothing outside the buffers is touched."""
    c = TreeCase(81, 4, 4, 128, 16, [9, 30], [40, 60])
    c.row_off = dev([9, 0, 39])
    o, lse = c.run(B)
    torch.cuda.synchronize()
    assert (c.obig == 7).all()
