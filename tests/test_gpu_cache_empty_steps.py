"""Steps that bring no row: requests that wait, end or lose drafts, and nothing else."""
import ctypes as C

import pytest
import torch

import paper_2402_02446_b200 as L
from cache_model import Tables
from paper_2402_02446_b200 import binding

DEV = "cuda:0"
E = binding.STATUS_NAMES.index
P = 4096


def _int(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


@pytest.mark.gpu
@pytest.mark.parametrize("commit", [True, False])
@pytest.mark.parametrize("added", [[0, 0, 0], [-3, 0, -50], [-60, -20, -50]])
def test_steps_without_rows(added, commit):
    model, pages = Tables(3, 8, 20, 16), L.new_page_table(3, 8, 20, 16, device=DEV)
    L.cache_step(pages, _int([60, 20, 50]), 130)
    model.step([60, 20, 50], 130, 130)
    before = pages.lengths.tolist()
    step = L.cache_step(pages, _int(added), 0, commit=commit)
    step = L.cache_step(pages, _int(added if not commit else [0, 0, 0]), 0, step=step, commit=commit)
    model.step(added, 0, 1)
    assert L.poll_status(step.buf) == 0
    assert step.slots.shape == step.positions.shape == (0,) and step.slots.dtype == torch.int32
    assert step.lengths.tolist() == model.lengths and step.ring.tolist() == model.ring and pages.free.tolist() == model.free
    assert pages.lengths.tolist() == (model.lengths if commit else before)
    # what a program does with a step's rows, for none
    for dtype in (torch.bfloat16, L.MXINT8):
        cache = L.new_kv_cache(20, 16, 2, 64, dtype=dtype, device=DEV)
        none = torch.empty((0, 2, 64), dtype=torch.bfloat16, device=DEV)
        launches = L.launch_count()
        L.append_kv(none, none, cache, step.slots)
        Y = L.paged_attention(torch.empty((0, 4, 64), dtype=torch.bfloat16, device=DEV), cache, pages, step)
        assert Y.shape == (0, 4, 64) and L.launch_count() == launches and not bool(cache.keys.any())


@pytest.mark.gpu
def test_rows_do_not_fit_such_a_step():
    pages = L.new_page_table(3, 8, 20, 16, device=DEV)
    step = L.cache_step(pages, _int([1, 0, 7]), 0)
    assert L.poll_status(step.buf) == E("LQER_ERR_BOUNDS") and step.lengths.tolist() == [0, 0, 0] and step.ring.tolist() == [0, 20]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, L.MXINT8])
@pytest.mark.parametrize("most", [1, 40, 1000])
@pytest.mark.parametrize("R", [1, 3, 50])
def test_rows_of_padding_alone(R, most, dtype):
    pages, cache = L.new_page_table(R, 8, 8 * R, 16, device=DEV), L.new_kv_cache(8 * R, 16, 2, 64, dtype=dtype, device=DEV)
    L.cache_step(pages, _int([37] * R), 37 * R)
    step = L.cache_step(pages, _int([0, -2, -37, 0, 0][:R] + [0] * (R - 5)), 40, max_added=most)
    assert step.slots.tolist() == step.positions.tolist() == [-1] * 40
    x = torch.ones((40, 2, 64), dtype=torch.bfloat16, device=DEV)
    L.append_kv(x, x, cache, step.slots)
    Y = torch.full((40, 8, 64), 7.0, dtype=torch.bfloat16, device=DEV)
    L.paged_attention(torch.ones_like(Y), cache, pages, step, Y=Y)
    assert L.poll_status(step.buf) == 0 and bool((Y == 7).all()) and not bool(cache.keys.any())


@pytest.mark.gpu
def test_in_a_graph():
    pages = L.new_page_table(2, 8, 20, 16, device=DEV)
    L.cache_step(pages, _int([60, 20]), 80)
    added = _int([-1, -1])
    step = L.cache_step(pages, added, 0)
    s = torch.cuda.Stream(DEV)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            L.cache_step(pages, added, 0, step=step)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert pages.lengths.tolist() == step.lengths.tolist() == [56, 16] and L.poll_status(step.buf) == 0


def test_refusals():
    def step(M, slots, positions, le=3 * P):
        table = C.byref(binding._Table(P, 2 * P, 4, 4, 8, 16))
        return L.lib().lqer_cache_step(table, le, 4 * P, 5 * P, M, 1, 6 * P, 7 * P, slots, positions, 10 * P, 1 << 20, None)

    # rows and lists go together: none of both, or some of both
    for slots, positions in ((8 * P, None), (None, 9 * P), (8 * P, 9 * P)):
        assert step(0, slots, positions) == E("LQER_ERR_SHAPE" if slots and positions else "LQER_ERR_NULL")
    assert step(1, None, None) == E("LQER_ERR_NULL") and step(-1, None, None) == E("LQER_ERR_NULL")
    assert step(0, None, None, le=None) == E("LQER_ERR_NULL") and step(0, None, None, le=P + 2) == E("LQER_ERR_ALIGN")
    pages = L.new_page_table(4, 4, 8, 16, device="cpu")
    with pytest.raises(ValueError):
        L.cache_step(pages, torch.zeros(4, dtype=torch.int32), -1)
