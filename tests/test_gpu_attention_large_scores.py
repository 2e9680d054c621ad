"""Scores of any size: a row's weights go by differences of scores, however large those are.

Queries and keys are small integers, so products and scores are exact, two scores differ by nothing or by one or more, and with a large scale only the
largest ones of a row weigh anything: those that share the top, all the same.  What is left of the bound is the rounding of weights, sums and results (cache_model.tolerance
without an error of the scores).

With scores far apart a row's result may be a tiny number: where its only weight of any size stands by a value of exactly 0.  A weight below 2^-126 counts as 0, and so may its
product with a value where that is below 2^-126, so that of `length` keys each may lose 2^-126 times its value's size, and once more 2^-126."""
import pytest
import torch

import paper_2402_02446_b200 as L
from cache_model import Batch, attention64, cache_values, tolerance

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16 = torch.bfloat16
# one row by several CTAs, drafts, tiles of rows, tiles divided over their keys
REQUESTS = [[(700, 1), (5, 1)], [(333, 8), (40, 2)], [(0, 300), (40, 1)], [(3000, 300)]]


def refill(b, K, V):
    """Other keys and values [tokens, heads, D] for all tokens of a batch, request by request."""
    page, slots = b.pages.page, []
    for r, (before, n) in enumerate(b.requests):
        j = torch.arange(before + n, device=DEV)
        slots.append(b.pages.tables[r, j // page] * page + (j % page).int())
    L.append_kv(K, V, b.cache, torch.cat(slots))


def check(b, Y, scale, window=0, sinks=0, exact=True):
    """exact: the scores have no error."""
    whole = cache_values(b.cache)
    row = 0
    for r, (before, n) in enumerate(b.requests):
        ids = b.pages.tables[r, :(before + n + b.pages.page - 1) // b.pages.page].long()
        K, V = (x[ids].transpose(0, 1).flatten(1, 2)[:, :before + n] for x in whole)
        y, weighed, most = attention64(b.Q[row:row + n].double(), K, V, n, window, sinks, scale)
        lost = (before + n) * 2.0 ** -126 * (1.0 + float(V.abs().max()))
        off = (Y[row:row + n].double() - y).abs() / (tolerance(y, weighed, 0.0 if exact else most, b.D, before + n) + lost)
        assert bool(torch.isfinite(Y[row:row + n]).all()), f"request {r}"
        assert float(off.max()) <= 1.0, (r, float(off.max()))
        row += n


@pytest.mark.parametrize("scale", [1e6, 1e9, -1e9, 3e15, 9e29])
@pytest.mark.parametrize("requests", REQUESTS)
@pytest.mark.parametrize("dtype,D", [(BF16, 128), (BF16, 64), (L.MXINT8, 128), (L.MXINT8, 64)])
def test_only_the_largest_scores_weigh_anything(dtype, D, requests, scale):
    b = Batch(requests, 8, 8, D, 16, dtype)
    g = torch.Generator(device=DEV).manual_seed(3)
    tokens = sum(x + n for x, n in requests)
    whole = lambda *s: torch.randint(-2, 3, s, generator=g, device=DEV).to(BF16)  # noqa: E731
    refill(b, whole(tokens, 8, D), torch.randn((tokens, 8, D), generator=g, device=DEV).to(BF16))
    b.Q = whole(b.M, 8, D)
    for window, sinks in ((0, 0), (200, 3)):
        Y = L.paged_attention(b.Q, b.cache, b.pages, b.step, window=window, sinks=sinks, scale=scale)
        assert L.poll_status(b.step.buf) == 0
        check(b, Y, scale, window, sinks)


@pytest.mark.parametrize("scale", [1.0, 10.0, -30.0])
@pytest.mark.parametrize("requests", REQUESTS)
@pytest.mark.parametrize("dtype", [BF16, L.MXINT8])
def test_scores_of_some_hundreds(dtype, requests, scale):
    b = Batch(requests, 8, 8, 128, 16, dtype)
    check(b, L.paged_attention(b.Q, b.cache, b.pages, b.step, scale=scale), scale, exact=False)
