"""The calls for requests with more than one continuation on a host without a GPU: refusals before any device work, and the 64-bit
definitions against hand-worked values."""
import math

import numpy as np
import pytest

from oracle import branching, serving


@pytest.fixture(scope="module")
def B():
    import __graft_entry__ as g
    g.build()
    from paper_2604_12782_b200 import binding
    return binding


def cache(B, **kw):
    a = dict(k=0x100000, v=0x200000, n_pages=4, page_size=16, n_heads=2, head_dim=128, page_stride=16 * 256, token_stride=256, head_stride=128)
    a.update(kw)
    return B.KvCacheStruct(*a.values())


def layers(B, *caches):
    return (B.KvCacheStruct * len(caches))(*caches)


def test_tree_mask_refusals(B):
    ok = dict(parents=0x1000, row=0x2000, base=0x3000, R=2, T=40, mask=0x4000, words=2, ld=2, pos=0x5000)

    def call(**kw):
        return B._lib.osc_tree_mask(*{**ok, **kw}.values(), None)
    for k in ("parents", "row", "mask"):
        assert call(**{k: None}) == -1, k
    assert call(T=0) == 0 and call(T=0, mask=None, parents=None) == 0
    assert call(R=-1) == -1 and call(T=-1) == -1
    assert call(words=0) == -2 and call(words=33, ld=33) == -2 and call(ld=1) == -2
    for out in ("mask", "pos"):
        for other in ("parents", "row", "base", "mask", "pos"):
            if out != other:
                assert call(**{out: ok[other]}) == -1, (out, other)
    assert call(pos=0x4000 + 39 * 8) == -1 and call(parents=0x4000 - 8) == -1 and call(base=0x4000 + 316) == -1


def test_tree_attention_refusals(B):
    ok = dict(Q=0x1000, T=4, ldq=512, n_q=4, c=cache(B), R=2, row=0x6000, kv=0x7000, table=0x8000, cols=3, ld=3, P=0, goff=None, plen=None, ptab=None,
              pcols=0, ldp=0, mask=0x9000, words=1, ldm=1, max_new=0, scale=0.1, O=0xA000, ldo=512, lse=None, ws=0x10000, n=1 << 40)

    def call(**kw):
        return B._lib.osc_tree_attention(*{**ok, **kw}.values(), None)
    assert call(T=0) == 0 and call(R=0) == 0
    for k in ("Q", "row", "kv", "table", "O", "ws", "mask"):
        assert call(**{k: None}) == -1, k
    assert call(words=0) == -2 and call(words=33, ldm=33) == -2 and call(words=2, ldm=1) == -2 and call(words=-1) == -2
    assert call(T=-1) == -1 and call(n_q=5) == -2 and call(c=cache(B, page_size=24)) == -2 and call(scale=math.nan) == -1 and call(ldq=516) == -4
    assert call(n=1000) == -5
    assert call(O=0x9000) == -1 and call(lse=0x9000) == -1 and call(mask=0x10000 + 128) == -1


def test_token_logprobs_refusals(B):
    ok = dict(x=0x100000, dtype=0, T=4, V=100, ld=100, scale=1.0, ids=0x1000, n_ids=2, ld_ids=2, lp=0x2000, lse=0x3000, ent=0x4000, k=3, tid=0x5000, tlp=0x6000)

    def call(**kw):
        return B._lib.osc_token_logprobs(*{**ok, **kw}.values(), None)
    for k in ("x", "ids", "lp", "tid", "tlp"):
        assert call(**{k: None}) == -1, k
    assert call(T=0) == 0 and call(T=0, x=None) == 0
    assert call(dtype=2) == -1 and call(dtype=-1) == -1 and call(T=-1) == -1 and call(V=0) == -1 and call(n_ids=-1) == -1 and call(k=-1) == -1
    for s in (0.0, -1.0, math.inf, math.nan, 2e30):
        assert call(scale=s) == -1, s
    assert call(k=33) == -2 and call(ld=99) == -2 and call(ld_ids=1) == -2 and call(x=0x100001) == -4 and call(x=0x100002, dtype=1) == -4
    for out in ("lp", "lse", "ent", "tid", "tlp"):
        for other in ("x", "ids", "lp", "lse", "ent", "tid", "tlp"):
            if out != other:
                assert call(**{out: ok[other]}) == -1, (out, other)
    assert call(lse=0x100000 + 2 * 399) == -1


def test_layer_refusals(B):
    def compact(ls, n=None, **kw):
        a = dict(R=2, row=0x1000, kv=0x2000, table=0x3000, cols=3, ld=3, keep=0x4000, kc=2, ldk=2, nk=0x5000, new=0x6000)
        return B._lib.osc_kv_compact(ls, len(ls) if n is None else n, *{**a, **kw}.values(), None)

    def copy(ls, n=None, a=0x1000, b=0x2000, used=0x3000, pages=2):
        return B._lib.osc_kv_copy_pages(ls, len(ls) if n is None else n, a, b, used, pages, None)
    c = cache(B)
    one = layers(B, c)
    for call in (compact, copy):
        assert call(one, 0) == -1 and call(None, 1) == -1 and call(one, -3) == -1
        for bad in (dict(k=None), dict(v=0x100000)):
            assert call(layers(B, c, cache(B, **bad))) == -1, bad
        for bad in (dict(n_pages=5), dict(page_size=32), dict(n_heads=4), dict(head_dim=64), dict(page_stride=8192), dict(token_stride=264), dict(head_stride=136)):
            assert call(layers(B, c, cache(B, **bad))) == -2, bad
        assert call(layers(B, c, cache(B, k=0x100008))) == -4 and call(layers(B, cache(B, head_dim=96))) == -2
    assert compact(one, R=0) == 0 and compact(one, R=-1) == -1 and compact(one, cols=-1) == -1 and compact(one, kc=-1) == -1
    for k in ("row", "kv", "table", "keep", "nk", "new"):
        assert compact(one, **{k: None}) == -1, k
    assert compact(one, ld=2) == -2 and compact(one, ldk=1) == -2 and compact(one, R=1 << 21) == -2
    for other in (0x1000, 0x1008, 0x2000, 0x3000 + 20, 0x4000, 0x5000 + 4):
        assert compact(one, new=other) == -1, hex(other)
    assert copy(one, pages=0) == 0 and copy(one, pages=-1) == -1 and copy(one, a=None) == -1 and copy(one, b=None) == -1 and copy(one, pages=(1 << 22) + 1) == -2
    assert copy(layers(B, cache(B, n_pages=0))) == 0


def test_trim_and_fork_refusals(B):
    okt = dict(a=0x1000, b=0x2000, R=2, page=16, table=0x3000, cols=3, ld=3, refs=0x4000, n_pages=8, freed=0x5000, n_freed=0x6000)

    def trim(**kw):
        return B._lib.osc_kv_trim(*{**okt, **kw}.values(), None)
    for k in ("a", "b", "table", "freed", "n_freed"):
        assert trim(**{k: None}) == -1, k
    assert trim(R=-1) == -1 and trim(cols=-1) == -1 and trim(n_pages=-1) == -1 and trim(page=0) == -2 and trim(ld=2) == -2 and trim(n_pages=13_000_000) == -2
    for out in ("table", "refs", "freed", "n_freed"):
        for other in ("a", "b", "table", "refs", "freed", "n_freed"):
            if out != other:
                assert trim(**{out: okt[other]}) == -1, (out, other)
    okf = dict(src=0x1000, dst=0x2000, n=2, len=0x3000, R=4, page=16, free=0x4000, n_free=3, table=0x5000, cols=3, ld=3, refs=0x6000, n_pages=8, ca=0x7000,
               cb=0x8000, cu=0x9000, taken=0xA000)

    def fork(**kw):
        return B._lib.osc_kv_fork(*{**okf, **kw}.values(), None)
    for k in ("src", "dst", "len", "free", "table", "ca", "cb", "cu", "taken"):
        assert fork(**{k: None}) == -1, k
    assert fork(n=-1) == -1 and fork(R=-1) == -1 and fork(cols=-1) == -1 and fork(n_free=-1) == -1 and fork(n_pages=-1) == -1
    assert fork(page=0) == -2 and fork(ld=2) == -2
    for out in ("len", "table", "refs", "ca", "cb", "cu", "taken"):
        for other in ("src", "dst", "len", "free", "table", "refs", "ca", "cb", "cu", "taken"):
            if out != other:
                assert fork(**{out: okf[other]}) == -1, (out, other)


def test_binding_refuses_wrong_tensors(B):
    import torch
    i, f, b = torch.zeros(4, dtype=torch.int32), torch.zeros(4), torch.zeros(4, 64, dtype=torch.bfloat16)
    m = i.view(2, 2)
    with pytest.raises(ValueError, match="cuda"):
        B.osc_tree_mask(i, i, None, m)
    with pytest.raises(ValueError, match="int32"):
        B.osc_tree_mask(i.long(), i, None, m)
    with pytest.raises(ValueError, match="float32"):
        B.osc_token_logprobs(b.half())
    with pytest.raises(ValueError, match="cuda"):
        B.osc_token_logprobs(b, lse=f)
    with pytest.raises(ValueError, match="int32"):
        B.osc_kv_trim(i.long(), i, 16, m, i, i, i)
    with pytest.raises(ValueError, match="cuda"):
        B.osc_kv_fork(i, i, i, 16, i, m, i, i, i, i, i)
    with pytest.raises(ValueError, match="no cache"):
        B.KvLayers([])


def test_definition_of_masks_by_hand():
    #      0
    #    1   2      4 (a second root)
    #    3          5, and 6 whose parent is not there
    bits, pos = branching.tree_mask([-1, 0, 0, 1, -1, 4, 9, 6], [0, 8], [100], 1)
    want = [[0], [0, 1], [0, 2], [0, 1, 3], [4], [4, 5], [], []]
    assert [np.nonzero(b)[0].tolist() for b in bits] == want and pos.tolist() == [100, 101, 101, 102, 100, 101, 0, 0]
    assert branching.packed(bits)[:, 0].tolist() == [1, 3, 5, 11, 16, 48, 0, 0]
    top = np.zeros((1, 64), bool)
    top[0, [31, 32]] = True
    assert branching.packed(top).tolist() == [[-2 ** 31, 1]]


def test_definition_of_attention_by_hand():
    rng = np.random.default_rng(0)
    q, k, v = rng.standard_normal((5, 2, 3, 8)), rng.standard_normal((9, 2, 8)), rng.standard_normal((9, 2, 8))
    chain = np.arange(9)[None] <= 4 + np.arange(5)[:, None]
    for x, y in zip(branching.attention(q, k, v, chain, 0.3), serving.attention(q, k, v, 5 + np.arange(5), 0.3)):
        assert np.allclose(x, y, rtol=1e-13)
    o, lse, _, _ = branching.attention(q, k, v, np.zeros((5, 9), bool), 0.3)
    assert (o == 0).all() and (lse == -np.inf).all()


def test_definition_of_logprobs_by_hand():
    x = np.log(np.array([[1.0, 2.0, 1.0, 4.0]]))
    lp, lse, ent, tid, tlp = branching.token_logprobs(x, [[1, 3, 4]], 1.0, 6)
    assert np.allclose(lp, [[math.log(0.25), math.log(0.5), -math.inf]]) and np.isclose(lse[0], math.log(8)) and np.isclose(ent[0], 1.75 * math.log(2))
    assert tid.tolist() == [[3, 1, 0, 2, -1, -1]] and np.allclose(tlp, [[math.log(0.5), math.log(0.25), math.log(0.125), math.log(0.125), -math.inf, -math.inf]])
    lp, lse, ent, tid, tlp = branching.token_logprobs(np.array([[-math.inf] * 3, [0.0, -math.inf, 0.0]]), [[0], [1]], 2.0, 2)
    assert lse[0] == -math.inf and ent[0] == 0 and tid.tolist() == [[0, 1], [0, 2]] and lp.tolist() == [[-math.inf], [-math.inf]]
    assert np.isclose(ent[1], math.log(2))


def test_definitions_of_moves_by_hand():
    cache = np.arange(12).reshape(3, 4, 1)           # pages of 4
    out, new_len = branching.kv_compact(cache, [0, 5], [8], np.array([[2, 0]]), np.array([[1, 4, 3]]), [3])
    # context 3 tokens on page 2; new tokens at places 3 .. 7: (2, 3), (0, 0) .. (0, 3); token 1 -> (2, 3), token 4 -> (0, 0); the list ends at 3
    assert out[2, 3, 0] == 0 and out[0, 0, 0] == 3 and out[0, 1:, 0].tolist() == [1, 2, 3] and new_len.tolist() == [5]
    table, refs, freed = branching.kv_trim([9, 4], [3, 0], 4, np.array([[5, 1, 2], [5, -1, -1]]), np.array([0, 1, 2, 0, 0, 2]), 6)
    assert table.tolist() == [[5, -1, -1], [-1, -1, -1]] and refs.tolist() == [0, 0, 1, 0, 0, 1] and freed.tolist() == [1]
    table, refs, length, copies, taken = branching.kv_fork([0, 0, 1], [2, 3, 4], np.array([6, 4, 0, 0, 0]), 4, [7, 8], np.array([[1, 2], [3, -1], [-1, -1], [-1, -1], [-1, -1]]),
                                                           np.array([0, 1, 1, 1, 0, 0, 0, 0, 0]), 9)
    assert table.tolist() == [[1, 2], [3, -1], [1, 7], [1, 8], [3, -1]] and refs.tolist() == [0, 3, 1, 2, 0, 0, 0, 1, 1]
    assert length.tolist() == [6, 4, 6, 6, 4] and copies.tolist() == [[2, 7, 2], [2, 8, 2], [-1, -1, 0]] and taken == 2


def test_keys_or_values_that_two_layers_share(B):
    """They would be moved twice.  (Copying a page twice does no harm.)"""
    def compact(ls):
        return B._lib.osc_kv_compact(ls, len(ls), 2, 0x1000, 0x2000, 0x3000, 3, 3, 0x4000, 2, 2, 0x5000, 0x6000, None)

    def many(n):
        return [cache(B, k=0x1000000 + i * 0x20000, v=0x1000000 + i * 0x20000 + 0x10000) for i in range(n)]
    for n in (2, 3, 36, 128, 129, 300):
        for a, b, plane in ((0, n - 1, "k"), ((n - 1) // 2, n - 1, "v"), (0, 1, "k")):
            ls = many(n)
            setattr(ls[b], plane, ls[a].k)
            assert compact(layers(B, *ls)) == -1 and b"another layer" in B._lib.osc_last_error(), (n, a, b, plane)
