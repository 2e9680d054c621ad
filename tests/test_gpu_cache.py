"""The tables of the paged cache from step to step against a plain model, and appending against the library's own quantiser."""
import random

import pytest
import torch

import paper_2402_02446_b200 as L
from cache_model import Tables
from paper_2402_02446_b200 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
E = binding.STATUS_NAMES.index


def _int(x, dtype=torch.int32):
    return torch.tensor(x, dtype=dtype, device=DEV)


def _compare(model, pages, step, want):
    slots, positions, status, plan = want
    assert L.poll_status(step.buf) == status
    assert step.slots.tolist() == slots and step.positions.tolist() == positions
    assert step.lengths.tolist() == model.lengths and step.ring.tolist() == model.ring
    assert pages.free.tolist() == model.free
    P = model.page
    for r, ln in enumerate(model.lengths):
        assert pages.tables[r, :(max(ln, 0) + P - 1) // P].tolist() == model.tables[r][:(max(ln, 0) + P - 1) // P]


@pytest.mark.parametrize("R,max_pages,n_pages,page", [(1, 4, 4, 16), (7, 9, 30, 16), (64, 40, 1500, 32), (1300, 6, 5000, 64), (33, 3, 40, 128)])
def test_steps_follow_the_model(R, max_pages, n_pages, page):
    rng = random.Random(R)
    model, pages = Tables(R, max_pages, n_pages, page), L.new_page_table(R, max_pages, n_pages, page, device=DEV)
    step = None
    for turn in range(12):
        added = []
        for r in range(R):
            ln, lot = model.lengths[r], rng.random()
            added.append(1 if turn % 3 else 0 if lot < 0.2 else -ln if lot < 0.3 else -rng.randint(0, 3) if lot < 0.4 else rng.randint(1, page * 2))
        M = max(1, sum(max(0, a) for a in added) + rng.choice((0, 5)))
        if step is not None and step.M != M:
            step = None
        step = L.cache_step(pages, _int(added), M, max_added=2 * page, step=step)
        _compare(model, pages, step, model.step(added, M, 2 * page))
    assert pages.lengths.tolist() == model.lengths and pages.ring.tolist() == model.ring


def test_a_step_that_is_not_committed_can_be_taken_again():
    model, pages = Tables(5, 8, 40, 16), L.new_page_table(5, 8, 40, 16, device=DEV)
    _compare(model, pages, L.cache_step(pages, _int([40, 100, 3, 0, 17]), 160), model.step([40, 100, 3, 0, 17], 160, 160))
    added = [1, -60, 30, 9, -17]
    before = pages.lengths.clone(), pages.ring.clone()
    step = L.cache_step(pages, _int(added), 41, commit=False)
    first = [t.clone() for t in (step.slots, step.positions, step.lengths, step.ring, pages.tables, pages.free)]
    assert torch.equal(pages.lengths, before[0]) and torch.equal(pages.ring, before[1])
    step = L.cache_step(pages, _int(added), 41, step=step, commit=False)
    assert all(torch.equal(a, b) for a, b in zip(first, (step.slots, step.positions, step.lengths, step.ring, pages.tables, pages.free)))
    _compare(model, pages, step, model.step(added, 41, 41))
    again = L.cache_step(pages, _int(added), 41)
    assert torch.equal(again.slots, first[0]) and torch.equal(pages.lengths, first[2]) and torch.equal(pages.ring, first[3])


def test_pages_that_come_back_serve_the_same_step():
    model, pages = Tables(2, 4, 4, 16), L.new_page_table(2, 4, 4, 16, device=DEV)
    _compare(model, pages, L.cache_step(pages, _int([64, 0]), 64), model.step([64, 0], 64, 64))
    _compare(model, pages, L.cache_step(pages, _int([-64, 60]), 64), model.step([-64, 60], 64, 64))


@pytest.mark.parametrize("added,M,most", [
    ([40, 40, 0, 40], 200, 200),      # too few pages from the third on, but not for those that need none
    ([1, 2, 3, 4], 6, 200),           # rows that do not fit
    ([5, 65, 1, 1], 200, 200),        # longer than a table
    ([5, 9, 1, 1], 200, 8),           # more than was said
    ([-5, -100, 2 ** 31 - 1, -2 ** 31], 30, 200),
])
def test_refusals_on_the_device(added, M, most):
    model, pages = Tables(4, 4, 8, 16), L.new_page_table(4, 4, 8, 16, device=DEV)
    start = [3, 16, 17, 0]
    _compare(model, pages, L.cache_step(pages, _int(start), 36), model.step(start, 36, 36))
    _compare(model, pages, L.cache_step(pages, _int(added), M, max_added=most), model.step(added, M, most))
    _compare(model, pages, L.cache_step(pages, _int([1, 1, 1, 1]), 4), model.step([1, 1, 1, 1], 4, 4))


@pytest.mark.parametrize("ring", [[5, 3], [-1, 2], [0, 9], [3, 11]])
def test_a_ring_that_cannot_be_refuses_what_moves_pages(ring):
    model, pages = Tables(3, 4, 8, 16), L.new_page_table(3, 4, 8, 16, device=DEV)
    _compare(model, pages, L.cache_step(pages, _int([20, 20, 5]), 45), model.step([20, 20, 5], 45, 45))
    model.ring = list(ring)
    pages.ring.copy_(_int(ring, torch.int64))
    added = [1, 20, -5]
    _compare(model, pages, L.cache_step(pages, _int(added), 30), model.step(added, 30, 30))


@pytest.mark.parametrize("tail", [2 ** 63 - 1, 2 ** 62])
def test_a_ring_at_the_end_of_its_type_is_one_that_cannot_be(tail):
    pages = L.new_page_table(2, 4, 8, 16, device=DEV)
    pages.lengths.copy_(_int([20, 20]))
    pages.ring.copy_(_int([tail - 4, tail], torch.int64))
    tables, free = pages.tables.clone(), pages.free.clone()
    step = L.cache_step(pages, _int([-20, 20]), 20)
    assert L.poll_status(step.buf) == E("LQER_ERR_BOUNDS")
    assert step.lengths.tolist() == [20, 20] and step.ring.tolist() == [tail - 4, tail]
    assert torch.equal(pages.tables, tables) and torch.equal(pages.free, free)


def test_entries_that_are_no_page_and_lengths_that_cannot_be():
    pages = L.new_page_table(3, 4, 8, 16, device=DEV)
    pages.lengths.copy_(_int([5, -1, 65]))
    pages.tables[0, 0] = 8
    step = L.cache_step(pages, _int([2, 1, -1]), 4)
    assert L.poll_status(step.buf) == E("LQER_ERR_BOUNDS")
    assert step.slots.tolist() == [-1] * 4 and step.lengths.tolist() == [7, -1, 65]
    pages = L.new_page_table(1, 4, 8, 16, device=DEV)
    pages.free.fill_(-7)
    step = L.cache_step(pages, _int([2]), 2)
    assert L.poll_status(step.buf) == E("LQER_ERR_BOUNDS") and step.slots.tolist() == [-1, -1]


def test_a_long_prompt_takes_a_launch_more():
    R, page, n = 3, 32, [20000, 0, 13007]
    model, pages = Tables(R, 700, 1200, page), L.new_page_table(R, 700, 1200, page, device=DEV)
    before = L.launch_count()
    step = L.cache_step(pages, _int(n), sum(n) + 100)
    assert L.launch_count() - before == 2
    _compare(model, pages, step, model.step(n, sum(n) + 100, sum(n) + 100))


def test_steps_in_a_graph_go_on():
    model, pages = Tables(6, 8, 48, 16), L.new_page_table(6, 8, 48, 16, device=DEV)
    added = _int([3, 0, 15, 1, 2, 1])
    step = L.cache_step(pages, added, 30, max_added=20)
    model.step([3, 0, 15, 1, 2, 1], 30, 20)
    s = torch.cuda.Stream(DEV)
    with torch.cuda.stream(s):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            L.cache_step(pages, added, 30, max_added=20, step=step)
    torch.cuda.synchronize()
    for new in ([3, 0, 15, 1, 2, 1], [1, 1, 1, 1, 1, 1], [-5, 20, -30, 4, 0, 1]):
        added.copy_(_int(new))
        graph.replay()
        torch.cuda.synchronize()
        _compare(model, pages, step, model.step(new, 30, 20))


@pytest.mark.parametrize("x", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dtype", [torch.bfloat16, L.MXINT8])
@pytest.mark.parametrize("M,hkv,D,page", [(1, 1, 64, 16), (7, 8, 128, 16), (201, 5, 64, 128), (1000, 2, 128, 32)])
def test_append(M, hkv, D, page, dtype, x):
    n_pages = (M + 50) // page + 2
    g = torch.Generator(device=DEV).manual_seed(M)
    cfg = L.default_config()
    cfg.a_bits = 6 if hkv == 5 else 8
    cache = L.new_kv_cache(n_pages, page, hkv, D, dtype=dtype, device=DEV)
    for t in (cache.keys, cache.values):
        t.copy_(torch.randint(0, 100, t.shape, generator=g, device=DEV))
    slots = torch.randperm(n_pages * page, generator=g, device=DEV)[:M].int()
    slots[M // 2:M // 2 + M // 10] = -1
    if M > 10:
        slots[0], slots[M - 1] = n_pages * page, -5
    both = (torch.randn((M, 4 * hkv * D + 16), generator=g, device=DEV) * torch.exp2(torch.randint(-9, 9, (M, 1), generator=g, device=DEV).float())).to(x)
    both[0, 3], both[M - 1, 5] = float("inf"), float("nan")
    K, V = both[:, 8:8 + hkv * D], both[:, 16 + hkv * D:16 + 2 * hkv * D].unflatten(1, (hkv, D))
    want = []
    for t, X in ((cache.keys, K), (cache.values, V)):
        w = t.clone()
        ok = ((slots >= 0) & (slots < n_pages * page)).nonzero()[:, 0]
        at, off = slots[ok].long() // page, slots[ok].long() % page
        rows = X[ok].reshape(len(ok), hkv, D)
        if dtype == L.MXINT8:
            m, e = L.quantize_activations(rows.float().reshape(-1, D).contiguous(), cfg=cfg)
            n = n_pages * hkv * page
            w[:n * D].view(torch.int8).view(n_pages, hkv, page, D)[at, :, off] = m.view(len(ok), hkv, D)
            w[n * D:].view(n_pages, hkv, page, D // 16)[at, :, off] = e.view(len(ok), hkv, D // 16)
        else:
            w[at, :, off] = rows.to(torch.bfloat16)
        want.append(w)
    L.append_kv(K, V, cache, slots, cfg=cfg)
    for t, w in zip((cache.keys, cache.values), want):
        assert torch.equal(t.view(torch.uint8), w.view(torch.uint8))
