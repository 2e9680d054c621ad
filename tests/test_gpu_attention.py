"""Attention over the paged cache against 64-bit arithmetic (the bound is derived in cache_model.tolerance), through tables and cache as a serving
program keeps them.  The cache holds NaN (bf16) or the largest numbers (MXINT8) wherever no token is."""
import numpy as np
import pytest
import torch

import paper_2402_02446_b200 as L
from cache_model import Batch, attention64, tolerance
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


@pytest.mark.parametrize("dtype", [BF16, L.MXINT8])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1500, 300)])
@pytest.mark.parametrize("requests,hq,hkv,D", [([(6000, 500), (0, 300), (9, 1)], 4, 2, 128), ([(3000, 1300)], 32, 8, 64), ([(2500, 700), (100, 620)], 20, 4, 128)])
def test_items_that_are_divided_over_their_keys(requests, hq, hkv, D, window, sinks, dtype, ratio_log):
    b = Batch(requests, hq, hkv, D, 32, dtype, pad=2)
    Y = _run(b, window, sinks, log=ratio_log)
    for _ in range(3):
        assert torch.equal(L.paged_attention(b.Q, b.cache, b.pages, b.step, window=window, sinks=sinks, Y=Y.clone()), Y)


@pytest.mark.parametrize("dtype", [BF16, L.MXINT8])
@pytest.mark.parametrize("hq,hkv,D", [(8, 8, 64), (16, 8, 128)])
def test_many_short_requests(hq, hkv, D, dtype, ratio_log):
    # so many that a warp takes a whole row
    _run(Batch([(i * 7 % 61, 1 + i % 3) for i in range(1400)], hq, hkv, D, 16, dtype, pad=2), log=ratio_log)


def test_narrower_mantissas_and_fp32_rows(ratio_log):
    cfg = L.default_config()
    cfg.a_bits, cfg.exp_min, cfg.exp_max = 6, -9, 4
    for requests in ([(90, 2), (33, 1)], [(90, 200), (0, 40)]):
        _run(Batch(requests, 8, 4, 128, 16, L.MXINT8, x_dtype=torch.float32, cfg=cfg), 50, 3, log=ratio_log)


@pytest.mark.parametrize("requests", [[(700, 1), (3, 1)], [(64, 4), (9, 1)], [(100, 300), (5, 1)]])
def test_views_streams_and_replays(requests):
    b = Batch(requests, 8, 2, 128, 16, pad=1)
    want = _run(b)
    # rows of a wider tensor, results off a 32-byte boundary, a given workspace
    wide = torch.zeros((b.M, 8 * 128 + 24), dtype=BF16, device=DEV)
    Q = wide[:, 8:8 + 8 * 128].unflatten(1, (8, 128))
    Q.copy_(b.Q)
    flat = torch.full((b.M * 8 * 128 + 8,), 7.0, dtype=BF16, device=DEV)
    Y = flat[8:].view(b.M, 8, 128)
    ws = torch.empty(L.attention_workspace_bytes(b.M, 8, b.cache, b.pages, b.step.max_added), dtype=torch.uint8, device=DEV)
    ws.fill_(0xFF)
    assert L.paged_attention(Q, b.cache, b.pages, b.step, Y=Y, ws=ws) is Y
    assert torch.equal(Y, want) and torch.all(flat[:8] == 7)
    # another stream
    s = torch.cuda.Stream(DEV)
    s.wait_stream(torch.cuda.current_stream())
    Z = L.paged_attention(b.Q, b.cache, b.pages, b.step, stream=s)
    torch.cuda.synchronize()
    n = sum(x for _, x in requests)
    assert torch.equal(Z[:n], want[:n])
    # a replay sees what the tensors hold then
    with torch.cuda.stream(s):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            L.paged_attention(Q, b.cache, b.pages, b.step, Y=Y, ws=ws)
    Q.copy_(-b.Q)
    torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    other = L.paged_attention(-b.Q, b.cache, b.pages, b.step)
    assert torch.equal(Y[:n], other[:n]) and not torch.equal(Y[:n], want[:n])


def test_generations_as_a_program_runs_them():
    """Two layers' caches under one table: prompts, decoding, drafts of which some are refused, a request that ends and one that takes its place; all through one
    captured step where the batch is decoding.  The attention of every step against 64 bits."""
    hq, hkv, D, page, R = 8, 2, 64, 16, 4
    pages = L.new_page_table(R, 12, 30, page, device=DEV)
    caches = [L.new_kv_cache(30, page, hkv, D, dtype=dt, device=DEV) for dt in (BF16, L.MXINT8)]
    g = torch.Generator(device=DEV).manual_seed(5)

    def step(added, M, most):
        plan = L.cache_step(pages, torch.tensor(added, dtype=torch.int32, device=DEV), M, max_added=most)
        for cache in caches:
            qkv = torch.randn((M, (hq + 2 * hkv) * D), generator=g, device=DEV).to(BF16)
            L.append_kv(qkv[:, hq * D:(hq + hkv) * D], qkv[:, (hq + hkv) * D:], cache, plan.slots)
            Q = qkv[:, :hq * D].unflatten(1, (hq, D))
            Y = L.paged_attention(Q, cache, pages, plan)
            assert L.poll_status(plan.buf) == 0
            b = Batch.__new__(Batch)
            b.requests = [(int(n) - max(a, 0), max(a, 0)) for n, a in zip(pages.lengths.tolist(), added)]
            b.hq, b.hkv, b.D, b.cfg, b.pages, b.cache, b.Q = hq, hkv, D, None, pages, cache, Q
            b.check(Y)

    step([40, 7, 0, 100], 150, 100)
    for _ in range(3):
        step([1, 1, 0, 1], 4, 1)
    step([4, 4, 0, 4], 12, 4)
    step([1, -2, 33, -int(pages.lengths[3])], 40, 33)      # drafts refused, one ends, one begins
    step([1, 1, 1, 60], 63, 60)                            # and its place is taken
    step([1, 1, 1, 1], 7, 1)
    held = sum((n + page - 1) // page for n in pages.lengths.tolist())
    ring = pages.ring.tolist()
    assert ring[1] - ring[0] == 30 - held
    free = [pages.free[i % 30].item() for i in range(ring[0], ring[1])]
    mine = [p for r in range(R) for p in pages.tables[r, :(pages.lengths[r] + page - 1) // page].tolist()]
    assert sorted(free + mine) == list(range(30))


@pytest.mark.parametrize("requests", [[(0, 130)], [(900, 100)], [(40, 1000), (3, 60)], [(300, 24)]])
@pytest.mark.parametrize("dtype", [BF16, L.MXINT8])
def test_the_output_projection_right_behind(dtype, requests):
    # the layer's kernels start while the attention's are still running, and use tensor memory of their own
    import lqer_inputs as gen
    spec = gen.LayerSpec("output", M=8, K=512, N=264, k=16, calib_rows=32, outlier_frac=0.01, outlier_scale=20.0, seed=78)
    A, B = gen.make_random_factors(spec)
    P = L.prepare_weights(*(torch.from_numpy(np.ascontiguousarray(v)).to(DEV) for v in (gen.make_weight(spec), A, B)))
    b = Batch(requests, 8, 8, 64, 16, dtype)
    ws = L.new_workspace(b.M, P)
    room = torch.empty(L.attention_workspace_bytes(b.M, 8, b.cache, b.pages, b.step.max_added), dtype=torch.uint8, device=DEV)
    Y = torch.empty((b.M, 8, 64), dtype=BF16, device=DEV)
    many = []
    for _ in range(20):
        L.paged_attention(b.Q, b.cache, b.pages, b.step, Y=Y, ws=room)
        many.append(L.linear_ex(Y.view(b.M, 512), P, ws))
    torch.cuda.synchronize()
    b.check(Y)
    want = L.linear_ex(Y.view(b.M, 512), P, ws)
    torch.cuda.synchronize()
    assert L.poll_status(b.step.buf) == 0 and L.poll_status(ws) == 0
    assert all(torch.equal(x, want) for x in many)
    P.release()


def test_plans_that_do_not_fit_write_nothing():
    b, other = Batch([(30, 2), (5, 1)], 8, 2, 64, 16), Batch([(30, 2), (5, 1), (1, 1)], 8, 2, 64, 16)
    long, wide = Batch([(30, 200), (5, 1)], 8, 2, 64, 16), Batch([(30, 200), (5, 1), (1, 1)], 8, 2, 64, 16)
    for mine, theirs in ((b, other), (long, wide)):
        Y = torch.full((mine.M, 8, 64), 7.0, dtype=BF16, device=DEV)
        theirs.step.M = mine.M                             # the binding is told otherwise: only the device can see
        L.paged_attention(mine.Q, mine.cache, mine.pages, theirs.step, Y=Y)
        assert L.poll_status(theirs.step.buf) == E("LQER_ERR_BAD_PACKED") and torch.all(Y == 7)


@pytest.mark.parametrize("dtype", [BF16, L.MXINT8])
@pytest.mark.parametrize("n", [1, 300])
def test_an_entry_that_is_no_page_is_reported(n, dtype):
    b = Batch([(40, n), (70, 1)], 8, 2, 64, 16, dtype)
    want = _run(b)
    b.pages.tables[0, 1] = 1 << 30
    Y = L.paged_attention(b.Q, b.cache, b.pages, b.step)
    assert L.poll_status(b.step.buf) == E("LQER_ERR_BOUNDS")
    assert torch.equal(Y[n:n + 1], want[n:n + 1])


def test_refused_requests_keep_their_rows():
    b = Batch([(20, 1), (30, 1), (10, 1)], 4, 1, 64, 16, spare=0)
    added = torch.tensor([1, 400, 1], dtype=torch.int32, device=DEV)
    step = L.cache_step(b.pages, added, 402)
    assert L.poll_status(step.buf) in (E("LQER_ERR_BOUNDS"), E("LQER_ERR_BUFFER_TOO_SMALL"))
    Q = torch.randn((402, 4, 64), device=DEV).to(BF16)
    Y = torch.full_like(Q, 7.0)
    L.append_kv(torch.zeros((402, 64), device=DEV), torch.zeros((402, 64), device=DEV), b.cache, step.slots)
    L.paged_attention(Q, b.cache, b.pages, step, Y=Y)
    assert torch.all(Y[1:401] == 7) and not torch.any(Y[0] == 7) and not torch.any(Y[401] == 7)


@pytest.mark.parametrize("dtype", [BF16, L.MXINT8])
def test_a_wait_that_runs_out(dtype):
    b = Batch([(100, 300), (0, 150)], 8, 2, 128, 16, dtype)
    want = _run(b)
    try:
        L.set_wait_limit_cycles(1_000_000)
        L.inject_stall(7)
        L.paged_attention(b.Q, b.cache, b.pages, b.step)
        assert L.poll_status(b.step.buf) == E("LQER_ERR_TIMEOUT")
    finally:
        L.inject_stall(-1)
        L.set_wait_limit_cycles(4_000_000_000)
    b.step.buf[:16].zero_()
    assert torch.equal(L.paged_attention(b.Q, b.cache, b.pages, b.step), want)


def test_results_are_the_same_every_time():
    for requests in ([(3000, 1), (17, 1), (900, 1)], [(3000, 3), (40, 1)], [(800, 300), (0, 77)]):
        b = Batch(requests, 16, 2, 128, 16)
        first = L.paged_attention(b.Q, b.cache, b.pages, b.step, window=700, sinks=2)
        for _ in range(5):
            assert torch.equal(L.paged_attention(b.Q, b.cache, b.pages, b.step, window=700, sinks=2), first)
    # a window that hides nothing is none
    assert torch.equal(L.paged_attention(b.Q, b.cache, b.pages, b.step, window=2 ** 31 - 1, sinks=2 ** 31 - 1), L.paged_attention(b.Q, b.cache, b.pages, b.step))


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("requests", [[(700, 1)], [(5000, 3)], [(300, 130)], [(1500, 140)]])
@pytest.mark.parametrize("D", [64, 128])
def test_scores_that_are_no_numbers_reach_the_rows_that_see_them(D, requests, bad):
    # in every column of a tile once: 16 heads times 8 tokens
    b = Batch(requests, 16, 16, D, 16)
    (before, n), = requests
    ids = b.pages.tables[0, :(before + n + 15) // 16].long()
    for k in range(8):
        keys = b.cache.keys.clone()
        for h in range(16):
            token = 16 * k + h
            b.cache.keys[ids[token // 16], h, token % 16, 0] = bad
        Y = L.paged_attention(b.Q, b.cache, b.pages, b.step).double()
        K, V = (x.double()[ids].transpose(0, 1).flatten(1, 2)[:, :before + n] for x in (b.cache.keys, b.cache.values))
        y = attention64(b.Q.double(), K, V, n, 0, 0, D ** -0.5)[0]
        assert torch.equal(torch.isnan(Y), torch.isnan(y)) and bool(torch.isnan(y).any())
        # an infinite score that is negative weighs nothing
        _, weighed, most = attention64(b.Q.double(), K.nan_to_num(0.0, 0.0, 0.0), V, n, 0, 0, D ** -0.5)
        good = ~torch.isnan(y)
        assert bool(((Y - y).abs() <= tolerance(y, weighed, most, D, before + n))[good].all())
        b.cache.keys.copy_(keys)


@pytest.mark.parametrize("requests,window,hidden,rows", [
    ([(0, 300)], 0, slice(150, 300), slice(0, 150)), ([(0, 700)], 0, slice(500, 700), slice(0, 500)), ([(1500, 140)], 0, slice(1600, 1640), slice(0, 100)),
    ([(0, 300)], 40, slice(0, 100), slice(139, 300)), ([(100, 8)], 0, slice(104, 108), slice(0, 4)), ([(2000, 8)], 500, slice(0, 1504), slice(4, 8)),
])
@pytest.mark.parametrize("D", [64, 128])
def test_hidden_values_weigh_nothing_however_large(D, requests, window, hidden, rows):
    b = Batch(requests, 8, 8, D, 16)
    (before, n), = requests
    want = L.paged_attention(b.Q, b.cache, b.pages, b.step, window=window)
    ids = b.pages.tables[0, :(before + n + 15) // 16].long()
    V = b.cache.values[ids].transpose(0, 1).flatten(1, 2)
    V[:, hidden] = 3e38
    b.cache.values[ids] = V.unflatten(1, (len(ids), 16)).transpose(0, 1)
    got = L.paged_attention(b.Q, b.cache, b.pages, b.step, window=window)
    assert torch.equal(got[rows], want[rows])
    others = torch.ones(n, dtype=torch.bool, device=DEV)
    others[rows] = False
    assert bool((got[others].abs() > 1e30).any())


@pytest.mark.parametrize("requests,hq,hkv", [([(5, 1), (90, 1)], 8, 2), ([(300, 1), (20, 2), (0, 5)], 32, 32), ([(700, 1)], 16, 2), ([(40, 8), (3, 8)], 1, 1)])
@pytest.mark.parametrize("most", [100, 5000])
def test_fewer_rows_than_a_request_might_bring(most, requests, hq, hkv, ratio_log):
    _run(Batch(requests, hq, hkv, 64, 16, max_added=most), log=ratio_log)
