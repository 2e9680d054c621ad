"""A scale of 0 weighs all that a row sees the same, whatever its scores: here they go to half the largest fp32 number."""
import pytest
import torch

import paper_2402_02446_b200 as L
from cache_model import Batch
from test_gpu_attention_large_scores import BF16, DEV, REQUESTS, check, refill

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("requests", REQUESTS)
def test_a_scale_of_zero_is_none_for_any_score(requests):
    b = Batch(requests, 8, 8, 64, 16)
    tokens = sum(x + n for x, n in requests)
    K, V = torch.zeros((tokens, 8, 64), device=DEV, dtype=BF16), torch.empty((tokens, 8, 64), device=DEV, dtype=BF16)
    sign = (1 - 2 * (torch.arange(tokens, device=DEV) % 2)).to(BF16)[:, None]
    K[:, :, 0] = sign * 1.75 * 2.0 ** 63
    V[:] = sign[:, :, None]                                # weights that go by the scores show in the sum at once
    refill(b, K, V)
    b.Q = torch.zeros((b.M, 8, 64), device=DEV, dtype=BF16)
    b.Q[:, :, 0] = 2.0 ** 63
    check(b, L.paged_attention(b.Q, b.cache, b.pages, b.step, scale=0.0), 0.0)
