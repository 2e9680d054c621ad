"""A row all of whose scores are minus infinity has no weights: the formula's 0 / 0, which is NaN, not a row of zeros."""
import pytest
import torch

import paper_2402_02446_b200 as L
from cache_model import Batch, attention64

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16
# a row by several CTAs, a row by one, a warp a row, drafts, tiles of rows, tiles divided over their keys
REQUESTS = [[(2000, 1), (3, 1)], [(0, 1)], [(4, 1)] * 700, [(0, 3), (20, 8)], [(0, 200), (30, 1)], [(3000, 300)]]


@pytest.mark.parametrize("requests", REQUESTS)
@pytest.mark.parametrize("D", [64, 128])
def test_rows_without_a_weight(D, requests):
    # infinite keys in a column: a row's scores are all infinite or all minus infinite, by the sign of its query there
    b = Batch(requests, 8, 8, D, 16)
    b.cache.keys[..., 0] = float("inf")
    Y = L.paged_attention(b.Q, b.cache, b.pages, b.step)
    assert L.poll_status(b.step.buf) == 0
    assert bool((b.Q[..., 0] < 0).any()) and bool(torch.isnan(Y).all())


@pytest.mark.parametrize("n", [1, 5, 150])
def test_a_first_key_of_the_other_sign(n):
    # the first token sees it alone; others have what else they see
    b = Batch([(0, n)], 8, 8, 64, 16)
    page = int(b.pages.tables[0, 0])
    b.cache.keys[page, :, 0, 0] = torch.where(b.Q[0, :, 0] > 0, float("-inf"), float("inf")).to(BF16)
    Y = L.paged_attention(b.Q, b.cache, b.pages, b.step).double()
    ids = b.pages.tables[0, :(n + 15) // 16].long()
    K, V = (x.double()[ids].transpose(0, 1).flatten(1, 2)[:, :n] for x in (b.cache.keys, b.cache.values))
    y = attention64(b.Q.double(), K, V, n, 0, 0, 64 ** -0.5)[0]
    assert bool(torch.isnan(Y[0]).all()) and torch.equal(torch.isnan(Y), torch.isnan(y))
