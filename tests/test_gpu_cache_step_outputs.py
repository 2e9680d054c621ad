"""What a step says of itself (lengths, ring) stays as it was when later steps go on from it."""
import pytest
import torch

import paper_2402_02446_b200 as L

DEV = "cuda:0"


def _int(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


@pytest.mark.gpu
@pytest.mark.parametrize("commit", [True, False])
def test_a_step_keeps_its_lengths_and_its_ring(commit):
    pages = L.new_page_table(3, 8, 20, 16, device=DEV)
    first = L.cache_step(pages, _int([20, 0, 5]), 25, commit=commit)
    assert first.lengths.tolist() == [20, 0, 5] and first.ring.tolist() == [3, 20]
    assert pages.lengths.tolist() == ([20, 0, 5] if commit else [0, 0, 0])
    second = L.cache_step(pages, _int([1, 40, -5]), 41)
    assert second.lengths.tolist() == ([21, 40, 0] if commit else [1, 40, 0])
    assert first.lengths.tolist() == [20, 0, 5] and first.ring.tolist() == [3, 20]
    assert pages.lengths.tolist() == second.lengths.tolist() and pages.ring.tolist() == second.ring.tolist()
    pages.lengths.zero_()
    assert second.lengths.tolist() == ([21, 40, 0] if commit else [1, 40, 0])


@pytest.mark.gpu
def test_refused_requests_stand_there_with_what_they_hold():
    pages = L.new_page_table(4, 4, 8, 16, device=DEV)
    pages.lengths.copy_(_int([5, -1, 65, 3]))
    step = L.cache_step(pages, _int([2, 1, -1, 1]), 4)
    assert step.lengths.tolist() == [7, -1, 65, 4] == pages.lengths.tolist()


@pytest.mark.gpu
def test_of_many_requests():
    R = 3000
    pages = L.new_page_table(R, 2, R, 16, device=DEV)
    added = torch.arange(R, dtype=torch.int32, device=DEV) % 3
    steps = [L.cache_step(pages, added, 3000, max_added=2) for _ in range(3)]
    for i, step in enumerate(steps):
        assert torch.equal(step.lengths, (i + 1) * added)
        assert step.ring.tolist() == [int((step.lengths > 0).sum()), R]


def test_sizes_on_the_host():
    pages = L.new_page_table(5, 4, 8, 16, device="cpu")
    from paper_2402_02446_b200.binding import CacheStep
    step = CacheStep(pages, 7, 1)
    assert step.lengths.shape == (5,) and step.lengths.dtype == torch.int32 and step.lengths.is_contiguous()
    assert step.ring.shape == (2,) and step.ring.dtype == torch.int64
    end = step.buf.data_ptr() + step.buf.numel()
    assert step.buf.data_ptr() <= step.ring.data_ptr() and step.lengths.data_ptr() + 20 <= end
