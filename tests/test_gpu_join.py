"""Attention calls without prefixes whose few tcgen05 units are cut into pieces over many CTAs, and calls that cut none because every request is small
while the caller has not said so (max_new = 0): what joins the pieces looks at all CTAs' cuts either way."""
import pytest
import torch

from branching_inputs import TreeCase
from serving_inputs import AttnCase

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2604_12782_b200 import binding
    return binding


@pytest.mark.parametrize("Hk,G,D,page,new,kv", [
    (8, 4, 128, 16, [100], [2000]),
    (8, 4, 128, 64, [300], [300]),
    (4, 4, 64, 32, [40] * 3, [2500, 700, 41]),
    (8, 4, 128, 16, [1] * 20 + [100], [500] * 21),
    (2, 8, 128, 64, [33], [9000]),
    (1, 1, 64, 16, [700], [700]),
    (3, 7, 128, 16, [60], [3001]),
    (8, 4, 128, 16, [130], [3000]),
    (8, 4, 128, 64, [1] * 30 + [200, 1, 70], [40] * 30 + [1500, 2, 900]),
    (4, 2, 64, 16, [64, 3, 90], [6000, 3, 500]),
])
def test_few_units_in_many_pieces(B, Hk, G, D, page, new, kv):
    assert sum(new) * G < 2048
    c = AttnCase(3, Hk, G, D, page, new, kv, tail_rows=2)
    c.check(*c.run(B), what="most new tokens not given")
    c.check(*c.run(B, max_new=max(new)))


@pytest.mark.parametrize("Hk,G,D,R,kv", [(8, 4, 128, 1, 600), (8, 4, 128, 30, 300), (2, 4, 64, 9, 5000), (1, 8, 128, 3, 40)])
def test_decoding_steps_that_are_not_announced(B, Hk, G, D, R, kv):
    c = AttnCase(4, Hk, G, D, 16, [1] * R, [kv + 13 * r for r in range(R)], tail_rows=1)
    c.check(*c.run(B))


@pytest.mark.parametrize("Hk,G,D,page,new,kv", [(8, 4, 128, 16, [140], [2500]), (2, 4, 64, 16, [60, 1, 33], [5000, 800, 33])])
def test_trees_in_many_pieces(B, Hk, G, D, page, new, kv):
    c = TreeCase(5, Hk, G, D, page, new, kv, tail_rows=1)
    c.check(*c.run(B, max_new=max(new)))
