"""Keys and values that no row of a step sees may hold anything, wherever they lie in a tile: between the first tokens and the window, and behind the end; also where
only the second of two row tiles sees the tile of keys in which they lie."""
import pytest
import torch

import paper_2402_02446_b200 as L
from cache_model import Batch

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.mark.parametrize("dtype", [BF16, L.MXINT8])
@pytest.mark.parametrize("requests,window,sinks", [
    ([(1000, 300)], 130, 3), ([(1000, 300), (77, 260)], 50, 0), ([(0, 129), (900, 129)], 64, 70), ([(300, 200), (333, 1), (2000, 4)], 40, 130), ([(128, 255)], 0, 0),
    ([(5000, 400)], 300, 20),
])
@pytest.mark.parametrize("hq,hkv,D", [(8, 8, 64), (8, 2, 128)])
def test_what_no_row_sees_may_hold_anything(hq, hkv, D, requests, window, sinks, dtype, ratio_log):
    b = Batch(requests, hq, hkv, D, 16, dtype, pad=2)
    want = L.paged_attention(b.Q, b.cache, b.pages, b.step, window=window, sinks=sinks)
    b.check(want, window, sinks, log=ratio_log)
    for r, (before, n) in enumerate(requests):
        j = torch.arange(before + n, device=b.dev)
        j = j[(j >= sinks) & (j <= before - window)] if window else j[:0]
        at, off = b.pages.tables[r, j // 16].long(), j % 16
        for t in (b.cache.keys, b.cache.values):
            if dtype == BF16:
                t[at, :, off] = float("nan")
            else:
                rows = b.cache.n_pages * hkv * 16
                t[:rows * D].view(-1, hkv, 16, D)[at, :, off] = 0x7F
                t[rows * D:].view(-1, hkv, 16, D // 16)[at, :, off] = 0xFF
    rows = sum(n for _, n in requests)
    for _ in range(3):
        assert torch.equal(L.paged_attention(b.Q, b.cache, b.pages, b.step, window=window, sinks=sinks)[:rows], want[:rows])
