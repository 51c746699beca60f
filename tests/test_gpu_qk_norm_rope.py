"""Norm and rotation of the heads and the write into the cache, against the 64-bit definition.

Tolerance of a turned channel: its two channels are normalised in fp32 (sum of at most 128 squares as a tree, rsqrt, three
products) and turned with a cosine and a sine off by at most 2^-22 each; 32 roundings of 2^-24 relative to |y_a| + |y_b|
cover it.  Then one rounding to bf16 (2^-8).  Channels that are only copied are equal bit for bit."""
import numpy as np
import pytest
import torch

from oracle import serving
from serving_inputs import BF16_HALF

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2604_12782_b200 import binding
    return binding


def run_case(B, seed, T, Hq, Hk, D, rot, axes=1, inter=False, far=4000, page=16, norm=True, layout="nhd", pad=0, in_place=False, scale=1.0,
             dense=False, stream=None, mul=1.5):
    rng = np.random.default_rng(seed)
    g = torch.Generator().manual_seed(seed)
    heads = Hq + 2 * Hk
    big = torch.full((T, heads * D + pad), float("nan"), dtype=torch.bfloat16)
    big[:, :heads * D] = torch.randn(T, heads * D, generator=g) * mul
    xb = big.cuda()
    x = big[:, :heads * D].double().numpy().reshape(T, heads, D)
    gq, gk = ((torch.rand(D, generator=g) + 0.5).to(torch.bfloat16) for _ in range(2))
    n = rot // 2
    inv = (1.0 / 1e6 ** (np.arange(n) / n)).astype(np.float32)
    axis = rng.integers(0, axes, n).astype(np.uint8) if axes > 1 else None
    pos = rng.integers(0, far, (axes, T)).astype(np.int32)
    n_pages = (T + 5) // page + 2
    slots = rng.permutation(n_pages * page)[:T].astype(np.int32)
    if dense:
        n_pages, page, slots = 1, T, np.arange(T, dtype=np.int32)
    elif T > 3:
        slots[T // 2] = -1
        slots[T // 3] = n_pages * page + 3        # a slot that the cache does not have
        slots[0] = -2 ** 31
    k, v = (torch.full((n_pages, page, Hk, D) if layout == "nhd" else (n_pages, Hk, page, D), 7.0, dtype=torch.bfloat16, device="cuda")
            for _ in range(2))
    if layout == "hnd":
        k, v = k.permute(0, 2, 1, 3), v.permute(0, 2, 1, 3)
    qbig = xb if in_place else torch.full((T, Hq * D + pad), 7.0, dtype=torch.bfloat16, device="cuda")
    B.osc_qk_norm_rope(xb[:, :heads * D], Hq, B.KvCache(k, v), qbig[:, :Hq * D], torch.from_numpy(pos if axes > 1 else pos[0]).cuda(),
                       B.Rope(torch.from_numpy(inv).cuda(), None if axis is None else torch.from_numpy(axis).cuda(), inter, scale),
                       gamma_q=gq.cuda() if norm else None, gamma_k=gk.cuda() if norm else None, eps=1e-6,
                       slots=None if dense else torch.from_numpy(slots).cuda(), stream=stream)
    torch.cuda.synchronize()

    def close(got, heads_x, gamma, what):
        ref, size = serving.qk_norm_rope(heads_x, gamma.double().numpy() if norm else None, 1e-6, inv, axis, pos, inter, scale)
        tol = BF16_HALF * np.abs(ref) + (1 + BF16_HALF) * 2.0 ** -19 * size + 1e-38
        err = np.abs(got - ref)
        assert (err <= tol).all(), f"{what}: {(err > tol).sum()} of {err.size} off, worst {np.max(err / tol)} of the tolerance"
    close(qbig[:, :Hq * D].float().cpu().numpy().astype(np.float64).reshape(T, Hq, D), x[:, :Hq], gq, "Q")
    live = (slots >= 0) & (slots < n_pages * page)
    kf, vf = (c.float().cpu().numpy().astype(np.float64).reshape(n_pages * page, Hk, D) for c in (k, v))
    if live.any():
        ref_k = np.zeros((T, Hk, D))
        ref_k[live] = kf[slots[live]]
        ref, size = serving.qk_norm_rope(x[:, Hq:Hq + Hk], gk.double().numpy() if norm else None, 1e-6, inv, axis, pos, inter, scale)
        tol = BF16_HALF * np.abs(ref) + (1 + BF16_HALF) * 2.0 ** -19 * size + 1e-38
        assert (np.abs(ref_k - ref) <= tol)[live].all(), "K"
        assert np.array_equal(vf[slots[live]], x[live][:, Hq + Hk:]), "V"
    rest = np.setdiff1d(np.arange(n_pages * page), slots[live])
    assert (kf[rest] == 7.0).all() and (vf[rest] == 7.0).all(), "slots of no token were written"
    if pad and not in_place:
        assert (qbig[:, Hq * D:] == 7.0).all()
    if in_place:
        tail = xb[:, Hq * D:heads * D].float().cpu().numpy().astype(np.float64).reshape(T, 2 * Hk, D)
        assert np.array_equal(tail, x[:, Hq:]), "K and V of QKV changed"


@pytest.mark.parametrize("T", [1, 2, 7, 33, 257, 1500])
def test_halves(B, T):
    run_case(B, T, T, 32, 8, 128, 128)


@pytest.mark.parametrize("Hq,Hk,D", [(1, 1, 64), (5, 1, 64), (7, 1, 128), (14, 2, 64), (32, 4, 128), (128, 8, 128), (3, 3, 128)])
def test_head_counts(B, Hq, Hk, D):
    run_case(B, Hq, 19, Hq, Hk, D, D)
    run_case(B, Hq + 1, 5000 // (Hq + 2 * Hk), Hq, Hk, D, D, page=64)


@pytest.mark.parametrize("D,rot", [(64, 16), (64, 32), (64, 48), (64, 64), (128, 16), (128, 48), (128, 64), (128, 112)])
@pytest.mark.parametrize("inter", [False, True])
def test_partial_and_interleaved(B, D, rot, inter):
    run_case(B, D + rot, 23, 6, 2, D, rot, inter=inter)


@pytest.mark.parametrize("axes", [2, 3])
@pytest.mark.parametrize("inter,rot", [(False, 128), (True, 128), (False, 64)])
def test_axes(B, axes, inter, rot):
    run_case(B, axes, 101, 8, 2, 128, rot, axes=axes, inter=inter)


def test_far_positions(B):
    run_case(B, 3, 200, 8, 2, 128, 128, far=2 ** 31 - 1)
    run_case(B, 4, 50, 4, 1, 64, 64, far=2_000_000, inter=True)


def test_options(B):
    run_case(B, 5, 60, 8, 2, 128, 128, norm=False)
    run_case(B, 6, 60, 8, 2, 128, 128, layout="hnd", pad=24)
    run_case(B, 7, 60, 8, 2, 128, 128, in_place=True)
    run_case(B, 8, 60, 8, 2, 128, 64, in_place=True)
    run_case(B, 9, 60, 8, 2, 128, 128, scale=1.25)
    run_case(B, 10, 60, 8, 2, 128, 128, dense=True)
    run_case(B, 11, 60, 8, 2, 64, 64, page=7)
    run_case(B, 12, 60, 8, 2, 128, 128, mul=1e-20)      # eps decides
    run_case(B, 13, 60, 8, 2, 128, 128, mul=1e15)
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        run_case(B, 14, 60, 8, 2, 128, 128)


def test_no_tokens_and_zero_rows(B):
    k = torch.full((2, 16, 2, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    v = k.clone()
    rope = B.Rope(torch.ones(32, device="cuda"))
    x = torch.zeros(3, 8 * 64, dtype=torch.bfloat16, device="cuda")
    q = torch.full((3, 4 * 64), 7.0, dtype=torch.bfloat16, device="cuda")
    pos = torch.zeros(3, dtype=torch.int32, device="cuda")
    g = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    B.osc_qk_norm_rope(x[:0], 4, B.KvCache(k, v), q[:0], pos[:0], rope, gamma_q=g, gamma_k=g)
    assert (k == 7).all() and (q == 7).all()
    B.osc_qk_norm_rope(x, 4, B.KvCache(k, v), q, pos, rope, gamma_q=g, gamma_k=g)      # x = 0: the norm's eps keeps it 0
    assert (q == 0).all() and (k[0, :3] == 0).all() and (k[0, 3:] == 7).all() and (k[1] == 7).all()


@pytest.mark.parametrize("T,inter", [(4735, False), (4736, False), (4741, False), (9473, False), (3600, True), (7104, True)])
def test_more_tokens_than_warps(B, T, inter):
    """About the numbers of tokens (warps on 148 SMs) behind which the rest is spread over several warps a token."""
    run_case(B, T, T, 3, 1, 64, 64, inter=inter)
    run_case(B, T + 1, T, 1, 1, 128, 128 if inter else 48, inter=inter)


@pytest.mark.parametrize("where", ["gap", "gap, other stride", "behind", "columns of a wider buffer"])
def test_queries_beside_qkv_in_one_buffer(B, where):
    """Queries in the gaps between QKV's rows, or right behind them: the same as in a buffer of their own."""
    T, Hq, Hk, D = 37, 4, 2, 128
    w, wq = (Hq + 2 * Hk) * D, Hq * D
    g = torch.Generator().manual_seed(3)
    data = torch.randn(T, w, generator=g).to(torch.bfloat16).cuda()
    pos = torch.arange(T, dtype=torch.int32, device="cuda") * 5
    rope = B.Rope((1e-4 ** (torch.arange(D // 2) / (D // 2))).cuda())
    gam = torch.ones(D, dtype=torch.bfloat16, device="cuda")

    def run(x, q):
        k, v = (torch.zeros(3, 16, Hk, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        B.osc_qk_norm_rope(x, Hq, B.KvCache(k, v), q, pos, rope, gamma_q=gam, gamma_k=gam)
        torch.cuda.synchronize()
        return q.clone(), k, v
    want = run(data, torch.zeros(T, wq, dtype=torch.bfloat16, device="cuda"))
    big = torch.full((4 * T * (w + wq),), 7.0, dtype=torch.bfloat16, device="cuda")
    if where == "behind":
        x, q = big[:T * w].view(T, w), big[T * w:T * (w + wq)].view(T, wq)
    elif where == "gap":
        x, q = (v[:, a:b] for v, a, b in ((big[:T * (w + wq)].view(T, -1), 0, w), (big[:T * (w + wq)].view(T, -1), w, w + wq)))
    elif where == "columns of a wider buffer":
        wide = big[:T * 2 * (w + wq)].view(T, -1)
        x, q = wide[:, wq + 8:wq + 8 + w], wide[:, :wq]
    else:
        x, q = big[:T * (w + wq)].view(T, -1)[:, :w], big[:2 * T * (w + wq)].view(T, -1)[:, w:w + wq]
    x.copy_(data)
    got = run(x, q)
    assert all(torch.equal(a, b) for a, b in zip(want, got)) and torch.equal(x, data)


def test_positions_with_a_stride(B):
    """Rows of positions further apart than there are tokens, as columns of a table of all steps: the same as side by side."""
    T, Hq, Hk, D = 45, 4, 2, 128
    g = torch.Generator().manual_seed(4)
    x = torch.randn(T, (Hq + 2 * Hk) * D, generator=g).to(torch.bfloat16).cuda()
    rope = B.Rope((1e-4 ** (torch.arange(D // 2) / (D // 2))).cuda(), (torch.arange(D // 2) % 3).to(torch.uint8).cuda())
    table = torch.randint(0, 9000, (3, T + 30), generator=g).to(torch.int32).cuda()
    out = []
    for pos in (table[:, 11:11 + T], table[:, 11:11 + T].contiguous()):
        k, v = (torch.zeros(4, 16, Hk, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        q = torch.zeros(T, Hq * D, dtype=torch.bfloat16, device="cuda")
        B.osc_qk_norm_rope(x, Hq, B.KvCache(k, v), q, pos, rope)
        out.append((q, k, v))
    assert all(torch.equal(a, b) for a, b in zip(*out))
    # and not by chance: other positions give other queries
    q = torch.zeros_like(q)
    B.osc_qk_norm_rope(x, Hq, B.KvCache(k, v), q, table[:, :T], rope)
    assert not torch.equal(q, out[0][0])
