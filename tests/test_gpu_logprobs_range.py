"""Scores at the ends of their ranges: scales so small that logits near the end of fp32's range count, rows that are sure of one token."""
import numpy as np
import pytest
import torch

from test_gpu_logprobs import B, DTYPES, call, check  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "f32"])
@pytest.mark.parametrize("V", [9, 1000, 40000, 151936])
@pytest.mark.parametrize("scale", [1e-19, 1e-20, 9e-21, 1e-30, 1e-35, 1e-36, 1e-37, 1e-38, 1e-40, 1e-44])
def test_small_scales(B, dtype, V, scale):                  # noqa: F811
    """Logits all over the type's range, largest next to lowest: differences, and sums of them, pass fp32's range where their products with the scale
    are ordinary numbers.  Scales below 10^-38 have fewer digits in fp32: the definition takes the scale that the call gets."""
    scale = float(np.float32(scale))
    g = torch.Generator().manual_seed(V)
    most = torch.finfo(dtype).max
    x = ((torch.rand(4, V, generator=g, dtype=torch.float64) * 2 - 1) * most).to(dtype).cuda()
    x[1, V // 2], x[1, 1] = most, -most
    x[2, V // 3:] = -most
    x[3, ::2] = -float("inf")
    check(B, x, np.tile(np.array([0, V - 1, V // 2]), (4, 1)), scale=scale, k=4)


@pytest.mark.parametrize("V", [1000, 3001, 70000])
@pytest.mark.parametrize("lead", [12.0, 16.0, 20.0, 40.0, 80.0])
def test_sure_rows_relative_to_their_size(B, V, lead):       # noqa: F811
    """One token `lead` ahead of equal others.  What is above 1 in l is summed by itself, so log probability and entropy are right relative to their own
    size: a term's exponent is lead log2 e with three roundings (4 2^-24 lead in e^-lead), exp2 is off by 2^-22, the sum of V positive terms by 2^-24 for each of
    at most V / 64 + 40 additions that a term goes through, logarithm, quotient and last sum by 2^-22.
    Where the others have 1 / 128 of the largest term or more (3000 of them at 12), l is summed with the 1: each of those additions rounds by 2^-24 of l, which
    is below 2, so ln l is off by at most 2 (V / 64 + 40) 2^-24, whatever its size, and S / l (lead at the most) by lead times that."""
    x = torch.zeros(1, V, device="cuda")
    x[0, 123] = lead
    got = call(B, x, [[123, 0]], k=1)
    rest = (V - 1) * np.exp(-lead)
    lp, ent = -np.log1p(rest), np.log1p(rest) + rest * lead / (1 + rest)
    rel = 4 * 2.0 ** -24 * lead + 2.0 ** -21 + (V / 64 + 40) * 2.0 ** -24
    assert got["top_ids"][0, 0] == 123
    one = 2 * (V / 64 + 40) * 2.0 ** -24 if rest >= 1 / 128 else 0.0
    assert rest < 1 and abs(got["logprob"][0, 0] - lp) <= rel * abs(lp) + one and abs(got["top_logprobs"][0, 0] - lp) <= rel * abs(lp) + one
    assert abs(got["entropy"][0] - ent) <= 2 * rel * ent + one * (1 + lead)


@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "f32"])
def test_a_very_long_row(B, dtype):                          # noqa: F811
    """2^27 logits: several thousand chunks to a block, parts of many chunks.  On its way into l a term goes through one addition for every chunk of its block
    (4096 values of fp32, an eighth of the row: V / 32768) and less than 100 others, each off by 2^-24; exponents and exp2 as in `tolerances`."""
    V = 2 ** 27 + 5
    x = torch.randn(1, V, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3)).mul_(3.0).to(dtype)
    got = call(B, x, [[0, V - 1, V // 3]], k=20)
    y = x[0].double()
    top = y.max()
    l = (y - top).exp().sum()
    lse = (top + l.log()).item()
    e_l = 120 * 2.0 ** -24 + 2.0 ** -22 + (V / 32768 + 100) * 2.0 ** -24
    assert abs(got["lse"][0] - lse) <= e_l + 2.0 ** -20
    assert np.abs(got["logprob"][0] - (y[torch.tensor([0, V - 1, V // 3], device="cuda")] - lse).cpu().numpy()).max() <= e_l + 2.0 ** -19
    ent = (l.log() - ((y - top).exp() * (y - top)).sum() / l).item()
    assert abs(got["entropy"][0] - ent) <= 3 * e_l * 20 + 2.0 ** -18
    best = x[0].float().topk(4000).values[19]
    at = torch.nonzero(x[0] >= best.to(dtype))[:, 0]
    order = at[torch.argsort(x[0, at].float(), descending=True, stable=True)][:20]
    assert got["top_ids"][0].tolist() == order.tolist()
