"""The calls around the paged key/value cache on a host without a GPU: refusals before any device work, and the 64-bit
definitions against hand-worked values."""
import ctypes as C
import math

import numpy as np
import pytest

from oracle import serving


@pytest.fixture(scope="module")
def B():
    import __graft_entry__ as g
    g.build()
    from paper_2604_12782_b200 import binding
    return binding


def cache(B, **kw):
    a = dict(k=0x1000, v=0x2000, n_pages=4, page_size=16, n_heads=2, head_dim=128, page_stride=16 * 256, token_stride=256, head_stride=128)
    a.update(kw)
    return B.KvCacheStruct(*a.values())


def test_kv_slots_refusals(B):
    ok = dict(cached=0x1000, fresh=0x2000, base=None, R=2, page=16, free=0x3000, n_free=4, table=0x4000, cols=3, ld=3, T=5, row=0x5000, kv=0x6000,
              slots=0x7000, pos=0x8000, taken=0x9000)

    def call(**kw):
        return B._lib.osc_kv_slots(*{**ok, **kw}.values(), None)
    for k in ("cached", "fresh", "free", "table", "row", "kv", "slots", "pos", "taken"):
        assert call(**{k: None}) == -1, k
    assert call(R=-1) == -1 and call(T=-1) == -1 and call(n_free=-1) == -1 and call(cols=-1) == -1
    assert call(page=0) == -2 and call(ld=2) == -2


def test_qk_norm_rope_refusals(B):
    def call(T=4, ld=8 * 128, n_q=4, c=None, rot=128, axes=1, pos=0x5000, Q=0x6000, ldq=512, qkv=0x7000, inv=0x8000, ld_pos=4, null_rope=False):
        r = B.RopeStruct(inv, None, rot, axes, 0, 1.0)
        return B._lib.osc_qk_norm_rope(qkv, T, ld, n_q, c or cache(B), None, None, 1e-6, None if null_rope else r, pos, ld_pos, None, Q, ldq, None)
    assert call(T=0) == 0 and call(T=0, qkv=None, Q=None, pos=None) == 0
    assert call(T=-1) == -1 and call(n_q=0) == -1 and call(null_rope=True) == -1
    assert call(qkv=None) == -1 and call(Q=None) == -1 and call(pos=None) == -1 and call(inv=None) == -1
    assert call(rot=8) == -2 and call(rot=20) == -2 and call(rot=144) == -2 and call(axes=0) == -1 and call(axes=4) == -1
    assert call(ld=1016) == -2 and call(ldq=504) == -2 and call(axes=2, ld_pos=3) == -2
    assert call(ld=1028) == -4 and call(ldq=516) == -4 and call(Q=0x6008) == -4 and call(qkv=0x7002) == -4
    assert call(c=cache(B, head_dim=96)) == -2 and call(c=cache(B, n_heads=0)) == -1 and call(c=cache(B, page_size=0)) == -1
    assert call(c=cache(B, k=None)) == -1 and call(c=cache(B, k=0x1008)) == -4 and call(c=cache(B, token_stride=252)) == -4
    assert call(c=cache(B, head_stride=64)) == -2 and call(c=cache(B, n_pages=2 ** 28)) == -2 and call(c=cache(B, n_pages=-1)) == -1


def test_paged_attention_refusals(B):
    ok = dict(Q=0x1000, T=4, ldq=512, n_q=4, c=cache(B), R=2, row=0x2000, kv=0x3000, table=0x4000, cols=3, ld=3, P=0, goff=None, plen=None, ptab=None,
              pcols=0, ldp=0, max_new=0, scale=0.1, O=0x5000, ldo=512, lse=None, ws=0x10000, n=1 << 40)

    def call(**kw):
        return B._lib.osc_paged_attention(*{**ok, **kw}.values(), None)
    assert call(T=0) == 0 and call(R=0) == 0
    for k in ("Q", "row", "kv", "table", "O", "ws"):
        assert call(**{k: None}) == -1, k
    pre = dict(P=2, goff=0x6000, plen=0x7000, ptab=0x8000, pcols=2, ldp=2)
    for k in ("goff", "plen", "ptab"):
        assert call(**{**pre, k: None}) == -1, k
    assert call(**{**pre, "ldp": 1}) == -2 and call(ld=2) == -2 and call(**{**pre, "pcols": -1}) == -1
    assert call(T=-1) == -1 and call(R=-1) == -1 and call(P=-1) == -1 and call(cols=-1) == -1 and call(max_new=-1) == -1
    assert call(n_q=5) == -2 and call(n_q=258, ldq=258 * 128, ldo=258 * 128) == -2 and call(n_q=0) == -1
    assert call(c=cache(B, page_size=24)) == -2 and call(c=cache(B, page_size=8)) == -2
    for s in (0.0, -1.0, math.inf, math.nan):
        assert call(scale=s) == -1, s
    assert call(ldq=504) == -2 and call(ldo=504) == -2 and call(ldq=516) == -4 and call(O=0x5004) == -4 and call(ws=0x10008) == -4
    assert call(n=1000) == -5
    sz = C.c_size_t()
    f = B._lib.osc_paged_attention_workspace_bytes
    assert f(1, 4, 128, 1, 0, C.byref(sz)) == 0 and sz.value > 0
    assert call(n=B.osc_paged_attention_workspace_bytes(4, 4, 128, 2, 0) - 1) == -5
    assert f(1, 4, 96, 1, 0, C.byref(sz)) == -2 and f(-1, 4, 128, 1, 0, C.byref(sz)) == -1 and f(1, 4, 128, 1, 0, None) == -1
    assert B.osc_paged_attention_workspace_bytes(300, 32, 128, 9, 2) > B.osc_paged_attention_workspace_bytes(200, 32, 128, 9, 2)


def test_overlapping_buffers_are_refused(B):
    """What one CTA reads another must not have written: every CTA of osc_kv_slots reads all lengths, a row of Q is read by several."""
    ok = dict(cached=0x1000, fresh=0x2000, base=0xA000, R=2, page=16, free=0x3000, n_free=4, table=0x4000, cols=3, ld=3, T=5, row=0x5000, kv=0x6000,
              slots=0x7000, pos=0x8000, taken=0x9000)

    def call(**kw):
        return B._lib.osc_kv_slots(*{**ok, **kw}.values(), None)
    for out in ("row", "kv", "slots", "pos", "taken", "table"):
        for other in ("cached", "fresh", "base", "free", "row", "kv", "slots", "pos", "taken", "table"):
            if out != other:
                assert call(**{out: ok[other]}) == -1, (out, other)
    assert call(kv=0x1004) == -1 and call(kv=0x1000 - 4) == -1 and call(taken=0x4000 + 5 * 4) == -1 and call(table=0x1000 - 5 * 4) == -1
    r = B.RopeStruct(0x8000, None, 128, 1, 0, 1.0)
    assert B._lib.osc_qk_norm_rope(0x7000, 4, 8 * 128, 4, cache(B), None, None, 1e-6, r, 0x5000, 4, None, 0x7000, 512, None) == -1
    sz = 1 << 40
    assert B._lib.osc_paged_attention(0x1000, 4, 512, 4, cache(B), 2, 0x2000, 0x3000, 0x4000, 3, 3, 0, None, None, None, 0, 0, 0, 0.1, 0x1000, 512, None,
                                      0x10000, sz, None) == -1


def test_binding_refuses_wrong_tensors(B):
    import torch
    i, b = torch.zeros(4, dtype=torch.int32), torch.zeros(2, 16, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="cuda"):
        B.osc_kv_slots(i, i, None, 16, i, i.view(2, 2), i, i, i, i, i)
    with pytest.raises(ValueError, match="int32"):
        B.osc_kv_slots(i.long(), i, None, 16, i, i.view(2, 2), i, i, i, i, i)
    with pytest.raises(ValueError, match="cuda"):
        B.KvCache(b, b)
    with pytest.raises(ValueError, match="bfloat16"):
        B.KvCache(b.half(), b.half())
    with pytest.raises(ValueError, match="float32"):
        B.Rope(torch.zeros(4, dtype=torch.float64))


def test_definition_of_slots_by_hand():
    # pages of 4; request 0 holds 3 tokens on page 7 and gets 2 (one on the old page, one on a new one), request 1 gets none,
    # request 2 starts with 5
    row, kv, table, slots, pos, taken = serving.kv_slots([3, 8, 0], [2, 0, 5], [10, 0, 100], 4, [20, 21, 22, 23],
                                                         [[7, -1], [1, 2], [-1, -1]], 8)
    assert row.tolist() == [0, 2, 2, 7] and kv.tolist() == [5, 8, 5] and taken == 3
    assert table.tolist() == [[7, 20], [1, 2], [21, 22]]
    assert slots.tolist() == [31, 80, 84, 85, 86, 87, 88, -1]
    assert pos.tolist() == [13, 14, 100, 101, 102, 103, 104, 0]


def test_definition_of_norm_and_rotation():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((3, 2, 16))
    g = rng.uniform(0.5, 1.5, 16)
    inv = np.array([1.0, 0.25, 0.125, 0.5, 0.0625, 0.75, 0.375, 0.03125], np.float32)
    pos = np.array([[0, 7, 100000]])
    y, size = serving.qk_norm_rope(x, g, 1e-6, inv, None, pos, False)
    n = x / np.sqrt((x * x).mean(-1, keepdims=True) + 1e-6) * g
    assert np.allclose(y[0], n[0], atol=1e-15)                                   # position 0 turns nothing
    assert np.allclose((y ** 2).sum(-1), (n ** 2).sum(-1), rtol=1e-13)           # a rotation keeps lengths
    z = (n[:, :, :8] + 1j * n[:, :, 8:]) * np.exp(1j * pos[0][:, None, None] * inv)
    assert np.allclose(y[:, :, :8], z.real, atol=1e-10) and np.allclose(y[:, :, 8:], z.imag, atol=1e-10)
    yi, _ = serving.qk_norm_rope(x, g, 1e-6, inv, None, pos, True)
    zi = (n[:, :, 0::2] + 1j * n[:, :, 1::2]) * np.exp(1j * pos[0][:, None, None] * inv)
    assert np.allclose(yi[:, :, 0::2], zi.real, atol=1e-10) and np.allclose(yi[:, :, 1::2], zi.imag, atol=1e-10)
    # two axes: pairs of axis 1 turn by the second row; the same position on both axes is the one-axis rotation
    ax = np.array([0, 1] * 4)
    two, _ = serving.qk_norm_rope(x, g, 1e-6, inv, ax, np.concatenate([pos, pos]), False)
    assert np.array_equal(two, y)
    two, _ = serving.qk_norm_rope(x, g, 1e-6, inv, ax, np.concatenate([pos, 0 * pos]), False)
    assert np.allclose(two[:, :, 1], n[:, :, 1]) and np.allclose(two[:, :, 0], y[:, :, 0])


def test_definition_of_attention():
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((3, 2, 4, 8)), rng.standard_normal((9, 2, 8)), rng.standard_normal((9, 2, 8))
    o, lse, absv, _ = serving.attention(q, k, v, [0, 1, 9], 0.5)
    assert (o[0] == 0).all() and np.isneginf(lse[0]).all()
    assert np.allclose(o[1], np.broadcast_to(v[0][:, None], (2, 4, 8)))
    for h in range(2):
        s = 0.5 * q[2, h] @ k[:, h].T
        w = np.exp(s) / np.exp(s).sum(-1, keepdims=True)
        assert np.allclose(o[2, h], w @ v[:, h]) and np.allclose(lse[2, h], np.log(np.exp(s).sum(-1)))
        assert (absv[2, h] >= np.abs(o[2, h])).all()


def test_qk_norm_rope_refuses_unaligned_gamma(B):
    """The norm's weights are read several channels at a time, so a view that begins inside such a group must not reach the kernel."""
    r = B.RopeStruct(0x8000, None, 128, 1, 0, 1.0)

    def call(gq, gk):
        return B._lib.osc_qk_norm_rope(0x70000, 4, 8 * 128, 4, cache(B), gq, gk, 1e-6, r, 0x5000, 4, None, 0x60000, 512, None)
    for off in (2, 4, 6, 8, 10, 14):
        assert call(0x9000 + off, None) == -4 and call(None, 0x9000 + off) == -4, off
        assert call(0x9000 + off, 0xA000) == -4 and call(0xA000, 0x9000 + off) == -4, off


def test_queries_that_overlap_qkv_without_being_it_are_refused(B):
    """Warps of one token, and steps of one warp, read heads of QKV after others have written queries, so only the same place can be
    read before it is written."""
    r = B.RopeStruct(0x800000, None, 128, 1, 0, 1.0)
    qkv, ld, T = 0x100000, 1024, 4                      # elements of two bytes; 4 query and 2 + 2 other heads of 128 channels

    def call(Q, ldq=512, T=T, ld=ld, qkv=qkv):
        return B._lib.osc_qk_norm_rope(qkv, T, ld, 4, cache(B), None, None, 1e-6, r, 0x900000, T, None, Q, ldq, None)
    for off in (16, 256, 512, 1024 - 16, 1024, 1536, 2048, 3 * 2048, 4 * 2048 - 16):     # bytes into QKV's 4 * 2048
        assert call(qkv + off) == -1 and call(qkv + off, ldq=ld) == -1, off
    for off in (16, 512, 3 * 1024 + 1008):              # QKV begins inside Q
        assert call(qkv - off) == -1, off
    assert call(qkv + 16, T=1) == -1 and call(qkv, ldq=520) == -1
    # rows of Q in the gaps of QKV's, of the same stride and of another: those that reach into a row
    assert call(qkv + 2048 + 1040, ldq=2048, ld=2048) == -1 and call(qkv + 2048 - 16, ldq=2048, ld=2048) == -1
    assert call(qkv + 2048, ldq=2560, ld=2048) == -1 and call(qkv + 2048 + 1040, ldq=4096, ld=2048) == -1
    assert call(qkv - 1024 + 16, ldq=2048, ld=2048) == -1 and call(qkv - 4096 - 1024, ldq=2560, ld=2048) == -1


def test_attention_outputs_that_overlap_anything_are_refused(B):
    """O, lse and the workspace are written while Q, the offsets and the tables are still read by other CTAs."""
    T, n_q, R, P, need = 4, 4, 2, 2, B.osc_paged_attention_workspace_bytes(4, 4, 128, 2, 2)
    base = 1 << 40                                       # (no address below zero where the workspace ends on a table)
    ok = dict(Q=base, T=T, ldq=512, n_q=n_q, c=cache(B), R=R, row=base + 0x200000, kv=base + 0x210000, table=base + 0x220000, cols=3, ld=3, P=P,
              goff=base + 0x230000, plen=base + 0x240000, ptab=base + 0x250000, pcols=2, ldp=2, max_new=0, scale=0.1, O=base + 0x300000, ldo=512,
              lse=base + 0x400000, ws=base + 0x1000000, n=need)

    def call(**kw):
        return B._lib.osc_paged_attention(*{**ok, **kw}.values(), None)
    rows = T * 1024
    for off in (0, 16, 512, 1024, rows - 16, -16, -512, 16 - rows):      # O against Q, rows of the same stride without gaps
        assert call(O=ok["Q"] + off) == -1, off
    # rows of Q and O of other strides and with gaps between them
    assert call(ldq=1024, ldo=1024, O=ok["Q"] + 1040) == -1 and call(ldq=1024, ldo=1024, O=ok["Q"] + 1008) == -1
    assert call(ldq=1024, ldo=2048, O=ok["Q"] + 1040) == -1 and call(ldq=1024, ldo=1536, O=ok["Q"] + 1024) == -1
    small = dict(row=4 * (R + 1), kv=4 * R, table=4 * R * 3, goff=4 * (P + 1), plen=4 * P, ptab=4 * P * 2)
    for name, size in small.items():
        assert call(O=ok[name] - rows + 16) == -1 and call(O=ok[name]) == -1, name
        assert call(lse=ok[name]) == -1 and call(lse=ok[name] + size - 4) == -1 and call(lse=ok[name] - 4 * T * n_q + 4) == -1, name
        assert call(ws=ok[name] - need // 16 * 16 + 16) == -1 and call(ws=ok[name]) == -1, name
    for name, size in (("Q", rows), ("O", rows)):
        assert call(lse=ok[name]) == -1 and call(lse=ok[name] + size - 4) == -1 and call(lse=ok[name] - 4 * T * n_q + 4) == -1, name
        assert call(ws=ok[name]) == -1 and call(ws=ok[name] + size - 16) == -1 and call(ws=ok[name] - need // 16 * 16 + 16) == -1, name
    assert call(lse=ok["ws"] + need - 4) == -1 and call(lse=ok["ws"]) == -1
    assert call(table=ok["ws"] + 4096, ld=100) == -1 and call(P=0, table=ok["O"] + 8) == -1
    for ld in (1 << 40, 1 << 62, (1 << 63) - 8):          # rows so far apart that the last ones have no address
        assert call(ldq=ld, O=ok["Q"] + 512) == -1 and call(ldo=ld, Q=ok["O"] + 512) == -1 and call(ld=ld, table=ok["ws"]) == -1, ld
        assert call(ldq=ld, ldo=ld, O=ok["Q"] + 512) == -1 and call(ldp=ld, ptab=ok["lse"]) == -1, ld


def test_one_place_for_keys_and_values_is_refused_where_they_are_written(B):
    r = B.RopeStruct(0x8000, None, 128, 1, 0, 1.0)

    def call(k, v):
        return B._lib.osc_qk_norm_rope(0x70000, 4, 8 * 128, 4, cache(B, k=k, v=v), None, None, 1e-6, r, 0x5000, 4, None, 0x60000, 512, None)
    assert call(0x1000, 0x1000) == -1
