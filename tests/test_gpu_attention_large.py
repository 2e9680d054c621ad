"""The cache and its attention at the far ends of their range: caches, queries and projections beyond 2^31 elements, a very long request, very many requests."""
import pytest
import torch

import paper_2402_02446_b200 as L
from cache_model import Batch, Tables

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16 = torch.bfloat16


@pytest.mark.parametrize("dtype", [BF16, L.MXINT8])
@pytest.mark.parametrize("requests", [[(300, 1), (40, 1)], [(200, 150), (40, 1)]])
def test_pages_beyond_two_billion_elements(requests, dtype, ratio_log):
    # 140000 pages of 16 tokens, 8 heads of 128: 2.3e9 elements; the requests hold the last ones
    b = Batch(requests, 16, 8, 128, 16, dtype, spare=140000, shuffle=False)
    assert b.cache.n_pages * 8 * 16 * 128 > 2 ** 31
    Y = L.paged_attention(b.Q, b.cache, b.pages, b.step)
    assert L.poll_status(b.step.buf) == 0
    used = b.pages.tables[:, 0]
    assert int(used.min()) > 139000
    b.check(Y, log=ratio_log, values=lambda ids: tuple(_rows(b, x, ids) for x in ("keys", "values")))


def _rows(b, name, ids):
    """The pages `ids` of the keys or values in 64 bits, without the rest of the cache."""
    x, c = getattr(b.cache, name), b.cache
    if c.dtype != L.MXINT8:
        return x[ids].double()
    n, shape = c.n_pages * c.kv_heads * c.page, (c.n_pages, c.kv_heads, c.page)
    m = x[:n * c.head_dim].view(torch.int8).view(*shape, c.head_dim)[ids].double()
    e = x[n * c.head_dim:].view(*shape, c.head_dim // 16)[ids].double()
    return m * torch.pow(2.0, e - 127 - 6).repeat_interleave(16, -1)


@pytest.mark.parametrize("n", [1, 60])
def test_queries_and_projections_beyond_two_billion_elements(n, ratio_log):
    R = 3000 // n
    b = Batch([(5, n)] * R, 4, 2, 64, 16)
    stride = 1 << 20
    rows = b.M
    far = torch.empty(rows * stride, dtype=BF16, device=DEV)
    Q = far.as_strided((rows, 4, 64), (stride, 64, 1))
    Q.copy_(b.Q)
    assert Q.stride(0) * (rows - 1) > 2 ** 31
    Y = L.paged_attention(Q, b.cache, b.pages, b.step)
    assert torch.equal(Y, L.paged_attention(b.Q, b.cache, b.pages, b.step))
    b.check(Y, log=ratio_log)
    K = far.as_strided((rows, 128), (stride, 1), 256)
    V = far.as_strided((rows, 128), (stride, 1), 512)
    K.copy_(torch.randn(rows, 128, device=DEV))
    V.copy_(torch.randn(rows, 128, device=DEV))
    L.append_kv(K, V, b.cache, b.step.slots)
    at = b.step.slots.long()
    assert torch.equal(b.cache.keys[at // 16, :, at % 16].flatten(1), K) and torch.equal(b.cache.values[at // 16, :, at % 16].flatten(1), V)


@pytest.mark.parametrize("window,sinks", [(0, 0), (70000, 100)])
def test_a_very_long_request(window, sinks, ratio_log):
    for n in (1, 130):
        b = Batch([(300000, n), (9, 1)], 4, 1, 64, 64)
        b.check(L.paged_attention(b.Q, b.cache, b.pages, b.step, window=window, sinks=sinks), window, sinks, log=ratio_log)


def test_very_many_requests():
    R = 16384
    model, pages = Tables(R, 2, 20000, 16), L.new_page_table(R, 2, 20000, 16, device=DEV)
    for added in ([i % 3 for i in range(R)], [1] * R, [-1 if i % 5 else 2 for i in range(R)]):
        M = sum(max(a, 0) for a in added) + 7
        step = L.cache_step(pages, torch.tensor(added, dtype=torch.int32, device=DEV), M, max_added=2)
        slots, positions, status, _ = model.step(added, M, 2)
        assert status == 0 and L.poll_status(step.buf) == 0
        assert step.slots.tolist() == slots and step.positions.tolist() == positions and pages.lengths.tolist() == model.lengths
        assert pages.free.tolist() == model.free and pages.ring.tolist() == model.ring
    # the values of a key head are its slots' numbers, so that with queries of zeros a row is the mean of those that it sees
    cache = L.new_kv_cache(20000, 16, 1, 64, device=DEV)
    numbers = (torch.arange(20000 * 16, device=DEV) % 251).to(BF16)
    cache.values.copy_(numbers.view(20000, 1, 16, 1).expand(-1, 1, 16, 64))
    step = L.cache_step(pages, torch.ones(R, dtype=torch.int32, device=DEV), R, max_added=1)
    assert L.poll_status(step.buf) == 0
    Y = L.paged_attention(torch.zeros((R, 2, 64), dtype=BF16, device=DEV), cache, pages, step)
    lengths, tables = pages.lengths.long(), pages.tables.long()
    j = torch.arange(32, device=DEV)
    seen = j < lengths[:, None]
    at = tables.clamp(min=0)[:, j // 16] * 16 + j % 16
    want = (numbers.double()[at] * seen).sum(1) / lengths
    assert float(((Y.double() - want[:, None, None]).abs() / want.clamp(min=1.0)[:, None, None]).max()) <= 2.0 ** -8 * 1.01
