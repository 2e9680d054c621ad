"""A table entry that is no page is reported when it is given back, too."""
import pytest
import torch

import paper_2402_02446_b200 as L
from paper_2402_02446_b200 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
E = binding.STATUS_NAMES.index


def _int(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("entry", [-1, 8, 2 ** 31 - 1, -2 ** 31])
@pytest.mark.parametrize("added", [[-40, 0], [-3, 0], [-40, 20]])
def test_entries_that_come_back(added, entry):
    pages = L.new_page_table(2, 4, 8, 16, device=DEV)
    L.cache_step(pages, _int([33, 2]), 35)
    pages.tables[0, 2] = entry
    step = L.cache_step(pages, _int(added), 20)
    assert L.poll_status(step.buf) == E("LQER_ERR_BOUNDS")
    # it comes back as it is: the ring's counts stay right, and whoever gets it finds out
    assert step.lengths.tolist() == [33 + added[0] if added[0] > -33 else 0, 2 + added[1]]
    back = 3 if added[0] == -40 else 1
    assert int(step.ring[1]) == 8 + back and int(pages.free[(8 + back - 1) % 8]) == entry


def test_good_entries_are_none():
    pages = L.new_page_table(2, 4, 8, 16, device=DEV)
    L.cache_step(pages, _int([64, 2]), 66)
    assert L.poll_status(L.cache_step(pages, _int([-64, 20]), 20).buf) == 0
