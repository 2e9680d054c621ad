"""Attention over the paged cache against 64-bit arithmetic (the bound is derived in cache_model.tolerance), through tables and cache as a serving
program keeps them.  The cache holds NaN (bf16) or the largest numbers (MXINT8) wherever no token is."""
import pytest
import torch

import paper_2402_02446_b200 as L
from cache_model import Batch
from paper_2402_02446_b200 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
E = binding.STATUS_NAMES.index
BF16 = torch.bfloat16


def _run(b, window=0, sinks=0, scale=None, log=None):
    left = torch.full((b.M, b.hq, b.D), 7.0, dtype=BF16, device=b.dev)
    Y = L.paged_attention(b.Q, b.cache, b.pages, b.step, window=window, sinks=sinks, scale=scale, cfg=b.cfg, Y=left.clone())
    assert L.poll_status(b.step.buf) == 0
    b.check(Y, window, sinks, scale, left, log)
    return Y


HEADS = [(32, 8, 128), (8, 8, 64), (10, 2, 128), (16, 1, 64), (5, 5, 128), (40, 2, 64)]


@pytest.mark.parametrize("dtype", [BF16, L.MXINT8])
@pytest.mark.parametrize("hq,hkv,D", HEADS)
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_one_new_token(page, hq, hkv, D, dtype, ratio_log):
    requests = [(0, 1), (15, 1), (16, 1), (700, 1), (5, 0), (0, 0), (63, 1), (64, 1), (65, 1), (2047, 1)]
    _run(Batch(requests, hq, hkv, D, page, dtype, pad=3), log=ratio_log)


@pytest.mark.parametrize("dtype", [BF16, L.MXINT8])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 4), (100, 0), (100, 200), (64, 64), (1000, 3), (5000, 1)])
def test_one_new_token_under_a_window(window, sinks, dtype, ratio_log):
    _run(Batch([(0, 1), (99, 1), (100, 1), (101, 1), (163, 1), (1023, 1), (3001, 1)], 16, 4, 128, 16, dtype), window, sinks, log=ratio_log)


@pytest.mark.parametrize("dtype", [BF16, L.MXINT8])
@pytest.mark.parametrize("window,sinks", [(0, 0), (3, 1), (40, 5)])
@pytest.mark.parametrize("hq,hkv,D", HEADS)
def test_a_few_new_tokens(hq, hkv, D, window, sinks, dtype, ratio_log):
    _run(Batch([(0, 3), (50, 8), (61, 5), (333, 1), (9, 0), (1000, 2)], hq, hkv, D, 16, dtype, pad=1), window, sinks, log=ratio_log)


@pytest.mark.parametrize("dtype", [BF16, L.MXINT8])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (7, 2), (128, 4), (200, 150)])
@pytest.mark.parametrize("hq,hkv,D", HEADS)
def test_prompts(hq, hkv, D, window, sinks, dtype, ratio_log):
    _run(Batch([(0, 129), (0, 1), (200, 300), (1, 77), (30, 0), (127, 128), (0, 260), (511, 3)], hq, hkv, D, 32, dtype, pad=9), window, sinks, log=ratio_log)


@pytest.mark.parametrize("scale", [0.0, -0.3, 2.0])
def test_other_scales(scale, ratio_log):
    for requests in ([(300, 1), (7, 1)], [(40, 150), (0, 20)]):
        _run(Batch(requests, 8, 2, 64, 16), scale=scale, log=ratio_log)


def test_a_long_request_beside_many_short_ones(ratio_log):
    _run(Batch([(30000, 1)] + [(3 * i % 40, 1) for i in range(300)], 8, 2, 128, 16), log=ratio_log)
    _run(Batch([(9000, 400), (12, 1), (0, 33)], 4, 2, 128, 64, max_added=400), log=ratio_log)
