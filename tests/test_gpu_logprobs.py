"""Log probabilities of given tokens, log-sum-exp, entropy and best alternatives against the 64-bit definition."""
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


def call(B, x, ids=None, scale=1.0, k=0, stream=None):
    T = x.shape[0]
    f = lambda *s: torch.full(s, 7.0, dtype=torch.float32, device="cuda")        # noqa: E731
    ids_t = torch.tensor(np.asarray(ids), dtype=torch.int32, device="cuda") if ids is not None else None
    out = dict(logprob=f(*ids_t.shape) if ids is not None else None, lse=f(T), entropy=f(T),
               top_ids=torch.full((T, k), 7, dtype=torch.int32, device="cuda") if k else None, top_logprobs=f(T, k) if k else None)
    B.osc_token_logprobs(x, ids_t, out["logprob"], scale=scale, lse=out["lse"], entropy=out["entropy"], top_ids=out["top_ids"],
                         top_logprobs=out["top_logprobs"], stream=stream)
    torch.cuda.synchronize()
    return {n: t.cpu().numpy().astype(np.float64) if t is not None else None for n, t in out.items()}


def tolerances(x, scale, lse):
    """Terms e^(scale d), d = x - max: the difference is rounded once (2^-24), its product with scale log2 e has two roundings and the constant one, so
    the exponent is off by at most a = 4 2^-24 |scale d|, against the largest that counts: terms with |scale d| > 30 add less than V e^-30.  exp2 itself is off by
    2^-22.  A thread adds V / 256 terms in two chains, 2^-24 a step, sixteen blocks and lanes join them: relative error of l below
    e_l = 4 2^-24 30 + 2^-22 + (V / 512 + 40) 2^-24.  lse and log probabilities: that, the logarithm's and the products' roundings (2^-22 of |scale max|, of
    |scale d| and of ln l).  Entropy: ln l by e_l, and S / l, the sum of |scale d| p, by 2 e_l of itself (at most ln V, or ln l)."""
    V = x.shape[1]
    e_l = 120 * 2.0 ** -24 + 2.0 ** -22 + (V / 512 + 40) * 2.0 ** -24 + V * 1e-13
    top = np.where(np.isfinite(x), np.abs(x), 0).max(-1) * scale
    return e_l + 2.0 ** -22 * (top + np.log(V) + 1), 3 * e_l * (np.log(V) + 1) + 2.0 ** -22 * np.log(V + 1)


def check(B, x, ids=None, scale=1.0, k=0, **kw):
    got = call(B, x, ids, scale, k, **kw)
    xd = x.double().cpu().numpy()
    lp, lse, ent, tid, tlp = branching.token_logprobs(xd, ids if ids is not None else np.zeros((x.shape[0], 0), int), scale, k)
    t_lse, t_ent = tolerances(xd, scale, lse)

    def close(a, b, tol, what):
        same = (np.isnan(a) & np.isnan(b)) | (np.isinf(b) & (a == b))
        with np.errstate(invalid="ignore"):
            bad = ~same & ~(np.abs(a - b) <= tol + 2.0 ** -22 * np.abs(np.where(np.isfinite(b), b, 0)))
        assert not bad.any(), f"{what}: {bad.sum()} off, worst {np.nanmax(np.where(bad, np.abs(a - b), 0))}, tolerance {np.max(tol)}"
    close(got["lse"], lse, t_lse, "lse")
    close(got["entropy"], ent, t_ent, "entropy")
    if ids is not None:
        close(got["logprob"], lp, t_lse[:, None], "logprob")
    if k:
        assert np.array_equal(got["top_ids"], tid), "top_ids"
        close(got["top_logprobs"], tlp, t_lse[:, None], "top_logprobs")


def rows(T, V, dtype, seed, mul=3.0, ld=None, at=0):
    """Logits whose rows begin `at` elements behind an aligned address and are ld apart; NaN around them."""
    g = torch.Generator().manual_seed(seed)
    ld = V if ld is None else ld
    buf = torch.full((at + T * ld + 16,), float("nan"), dtype=dtype, device="cuda")
    x = buf[at:at + T * ld].view(T, ld)[:, :V]
    x.copy_((torch.randn(T, V, generator=g) * mul).to(dtype))
    return x


DTYPES = [torch.bfloat16, torch.float32]


@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "f32"])
@pytest.mark.parametrize("T,V,k", [(1, 1, 1), (1, 2, 5), (3, 7, 7), (2, 8, 8), (5, 9, 3), (1, 255, 20), (4, 257, 32), (2, 2047, 1), (3, 2049, 8), (1, 16384, 20),
                                   (2, 16385, 20), (1, 33333, 5), (1, 151936, 20), (26, 32001, 5), (300, 4099, 4), (1000, 1000, 2)])
def test_shapes(B, dtype, T, V, k):
    ids = np.random.default_rng(V).integers(0, V, (T, 3))
    check(B, rows(T, V, dtype, V), ids, k=k)


@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "f32"])
@pytest.mark.parametrize("T,V,k", [(2, 262144, 32), (17, 200001, 1), (30, 151937, 20), (60, 131073, 0), (120, 99999, 8), (250, 65537, 5)])
def test_rows_over_clusters(B, dtype, T, V, k):
    """Rows of several chunks to a block, on clusters of eight, four, two and one."""
    check(B, rows(T, V, dtype, V), np.random.default_rng(V).integers(0, V, (T, 2)), k=k)


@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "f32"])
@pytest.mark.parametrize("at,pad", [(0, 1), (1, 0), (3, 5), (7, 2), (5, 8), (2, 3)])
def test_rows_at_any_element(B, dtype, at, pad):
    for V in (5, 100, 20000):
        check(B, rows(5, V, dtype, at, ld=V + pad, at=at), np.random.default_rng(1).integers(0, V, (5, 1)), k=4)


@pytest.mark.parametrize("scale", [0.01, 0.5, 1.0, 1.7, 30.0])
def test_temperatures(B, scale):
    for dtype in DTYPES:
        check(B, rows(4, 5000, dtype, 5), np.arange(12).reshape(4, 3), scale=scale, k=6)


@pytest.mark.parametrize("k", [0, 1, 2, 31, 32])
def test_numbers_of_alternatives(B, k):
    for T, V in ((1, 70000), (700, 3000)):
        check(B, rows(T, V, torch.bfloat16, k, mul=1.0), None, k=k)


@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "f32"])
@pytest.mark.parametrize("V", [10, 3000, 40000])
def test_equal_logits_and_rows_in_order(B, dtype, V):
    """Ties go to the lowest index; rows that rise or fall; rows with two values."""
    x = rows(7, V, dtype, 1)
    x[0] = 2.5
    x[1] = torch.linspace(-9, 9, V)
    x[2] = torch.linspace(9, -9, V)
    x[3] = torch.where(torch.arange(V) % 3 == 1, 1.0, -1.0)
    x[4] = torch.where(torch.arange(V) >= V - 5, 4.0, torch.linspace(-20, 0, V))
    x[5] = 0.0
    x[5, ::2] = -0.0
    x[6] = (torch.arange(V) // 700 * 0.5).to(dtype)
    check(B, x, np.tile(np.array([0, V - 1, V // 2]), (7, 1)), k=20)


@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "f32"])
@pytest.mark.parametrize("V", [9, 4000, 50000])
def test_masked_logits(B, dtype, V):
    """-inf and the type's lowest value, some, most, all but one, and all of a row."""
    inf, low = float("inf"), torch.finfo(dtype).min
    x = rows(8, V, dtype, 2)
    x[0, V // 2:] = -inf
    x[1, :V - 1] = -inf
    x[2] = -inf
    x[3] = low
    x[4, V // 3:] = low
    x[5, 1:] = low
    x[6] = -inf
    x[6, 3], x[6, V - 1] = -4.0, low
    x[7, ::2] = -inf
    check(B, x, np.tile(np.array([0, V - 1, 3]), (8, 1)), k=5)


@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "f32"])
def test_nan_and_inf(B, dtype):
    for V in (12, 3000):
        x = rows(5, V, dtype, 3)
        x[0, 5] = float("nan")
        x[1, 2] = float("inf")
        x[2] = float("nan")
        x[3, :] = -float("inf")
        x[3, 4] = float("nan")
        got = call(B, x, [[0, 5, 2]] * 5, k=4)
        for r in range(4):
            assert np.isnan(got["lse"][r]) and np.isnan(got["entropy"][r]) and np.isnan(got["logprob"][r]).all() and np.isnan(got["top_logprobs"][r]).all(), r
        check(B, x[4:], [[0, 5, 2]], k=4)
        xd = x.double().cpu().numpy()
        for r in range(4):                    # by value, NaN last, then by index
            want = sorted(range(V), key=lambda i: (np.isnan(xd[r, i]), 0 if np.isnan(xd[r, i]) else -xd[r, i], i))[:4]
            assert got["top_ids"][r].tolist() == want, r


def test_sure_rows_keep_their_digits(B):
    """One token far ahead: entropy and log probability are tiny, and nothing cancels beyond the rounding of l, which is just above 1.

    l is a sum in fp32, so each addition that the large term goes through is off by at most 2^-24 (half a step of numbers in 1 .. 2).  There are 17 of
    them for 1000 logits in fp32: two in the thread's chain (a vector of four in two chains), one that joins the chains, one onto the thread's sum, five over the
    warp, eight over the warps.  The logarithm and the last subtraction: 2^-23 of the result, 1e-6 of it with what exp2 is off by (2^-22)."""
    for lead in (12.0, 16.0, 20.0, 40.0):
        x = torch.zeros(1, 1000, device="cuda")
        x[0, 123] = lead
        got = call(B, x, [[123, 0]], k=1)
        rest = 999 * np.exp(-lead)
        p = 1 / (1 + rest)
        lp, ent = -np.log1p(rest), np.log1p(rest) + p * rest * lead
        assert abs(got["logprob"][0, 0] - lp) <= 17 * 2.0 ** -24 + 1e-5 * abs(lp)
        assert abs(got["entropy"][0] - ent) <= 17 * 2.0 ** -24 + 1e-5 * ent


@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "f32"])
@pytest.mark.parametrize("V", [3000, 70000, 300000])
def test_few_tokens_allowed(B, dtype, V):
    """All but a few logits masked, fewer than the alternatives asked for: the masked ones follow by index."""
    rng = np.random.default_rng(V)
    for n in (1, 5, 19, 40, 600):
        x = torch.full((2, V), -float("inf"), dtype=dtype, device="cuda")
        at = rng.choice(V, n, replace=False)
        x[0, at] = torch.randn(n, generator=torch.Generator().manual_seed(n)).to(dtype).cuda()
        x[1, at] = 0.5
        got = call(B, x, [[int(at[0]), 7]] * 2, k=20)
        for r in range(2):
            v = x[r].double().cpu().numpy()
            order = np.lexsort((np.arange(V), -v))[:20]
            assert got["top_ids"][r].tolist() == order.tolist()
            lse = np.log(np.exp(v[at]).sum())
            there = np.isfinite(v[order])
            assert abs(got["lse"][r] - lse) < 1e-5 and np.abs(got["top_logprobs"][r][there] - v[order][there] + lse).max() < 1e-5
            assert (got["top_logprobs"][r][~there] == -np.inf).all()


@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "f32"])
@pytest.mark.parametrize("V", [7, 300, 4001, 33000, 152064])
def test_very_sure_rows(B, dtype, V):
    """Where one token has nearly all of the probability, ln l = ln(1 + r), and r is summed without the 1.  Relative to its own size r is off as any sum of
    exponentials is (e_l in `tolerances`, here with |scale d| up to 60), and so are the log probability and the entropy, r (1 + lead) and less."""
    for lead in (9.0, 14.0, 25.0, 40.0):
        x = rows(4, V, dtype, V, mul=1.0, ld=V + 3, at=1)
        best = np.array([0, V - 1, V // 2, V // 3])
        x[torch.arange(4), torch.from_numpy(best)] = lead + np.log(V)
        got = call(B, x, best[:, None], k=2)
        xd = x.double().cpu().numpy()
        d = xd - xd[np.arange(4), best][:, None]
        d[np.arange(4), best] = -np.inf
        with np.errstate(invalid="ignore"):
            r = np.exp(d).sum(1)
            s = np.where(np.isfinite(d), np.exp(d) * d, 0).sum(1)
        rel = 4 * 60 * 2.0 ** -24 + 2.0 ** -21 + (V / 512 + 60) * 2.0 ** -24
        assert np.array_equal(got["top_ids"][:, 0], best)
        assert (np.abs(got["logprob"][:, 0] + np.log1p(r)) <= rel * np.log1p(r)).all(), (got["logprob"][:, 0], -np.log1p(r))
        ent = np.log1p(r) - s / (1 + r)
        assert (np.abs(got["entropy"] - ent) <= 2 * rel * ent).all(), (got["entropy"], ent)


def test_ids_outside_and_parts_left_out(B):
    x = rows(3, 500, torch.float32, 4)
    got = call(B, x, [[-1, 500, 2 ** 31 - 1], [0, 499, -2 ** 31], [7, 7, 7]])
    assert (got["logprob"][0] == -np.inf).all() and got["logprob"][1, 2] == -np.inf and np.isfinite(got["logprob"][1, :2]).all()
    assert got["logprob"][2, 0] == got["logprob"][2, 1]
    lse = torch.zeros(3, device="cuda")
    B.osc_token_logprobs(x, lse=lse)
    assert np.array_equal(lse.cpu().numpy(), got["lse"].astype(np.float32))
    wide = torch.full((3, 9), -1, dtype=torch.int32, device="cuda")
    wide[:, :2] = 3
    out = torch.zeros(3, 2, device="cuda")
    B.osc_token_logprobs(x, wide[:, :2], out)
    assert torch.allclose(out[:, 0], x[:, 3] - lse, atol=1e-5)
    many = torch.arange(500, device="cuda", dtype=torch.int32).repeat(3, 1)
    out = torch.zeros(3, 500, device="cuda")
    B.osc_token_logprobs(x, many, out)
    assert torch.allclose(out, x - lse[:, None], atol=1e-5)
    B.osc_token_logprobs(torch.zeros(0, 500, device="cuda"), lse=torch.zeros(0, device="cuda"))


def test_repeats_are_equal_and_streams(B):
    x = rows(40, 30000, torch.bfloat16, 6)
    a = call(B, x, np.zeros((40, 1), int), k=9)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for _ in range(3):
            b = call(B, x, np.zeros((40, 1), int), k=9)
            assert all(np.array_equal(a[n], b[n]) for n in a)
    lse, tid, tlp = torch.zeros(40, device="cuda"), torch.zeros(40, 9, dtype=torch.int32, device="cuda"), torch.zeros(40, 9, device="cuda")
    y = x.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.osc_token_logprobs(y, lse=lse, top_ids=tid, top_logprobs=tlp)
    for seed in (7, 8):
        y.copy_(rows(40, 30000, torch.bfloat16, seed))
        g.replay()
        torch.cuda.synchronize()
        want = call(B, y, k=9)
        assert np.array_equal(tid.cpu().numpy(), want["top_ids"]) and np.array_equal(lse.cpu().numpy(), want["lse"].astype(np.float32))


def test_logits_past_31_bits(B):
    """Rows whose offsets pass 2^31 elements."""
    V, T = 262144, 8200
    x = torch.empty(T, V, dtype=torch.bfloat16, device="cuda")
    x.fill_(-1.0)
    x[T - 1, 77], x[T - 1, V - 1], x[0, 5] = 9.0, 8.0, 7.0
    lse, tid, tlp = torch.zeros(T, device="cuda"), torch.zeros(T, 2, dtype=torch.int32, device="cuda"), torch.zeros(T, 2, device="cuda")
    B.osc_token_logprobs(x, lse=lse, top_ids=tid, top_logprobs=tlp)
    assert tid[T - 1].tolist() == [77, V - 1] and tid[0].tolist() == [5, 0] and tid[T - 2].tolist() == [0, 1]
    flat = np.log(V) - 1
    assert abs(lse[T - 2].item() - flat) < 1e-4 and abs(lse[T - 1].item() - np.log((V - 2) * np.exp(-1) + np.exp(9) + np.exp(8))) < 1e-4
