"""A quantised cache is read in the format in which it was written, and is not written in two."""
import pytest
import torch

import paper_2402_02446_b200 as L
from cache_model import Batch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _format(bits):
    cfg = L.default_config()
    cfg.a_bits = bits
    return cfg


@pytest.mark.parametrize("requests", [[(90, 2), (33, 1)], [(90, 200), (0, 40)]])
@pytest.mark.parametrize("bits", [4, 6, 8])
def test_attention_takes_the_format_of_the_cache(bits, requests):
    b = Batch(requests, 8, 4, 128, 16, L.MXINT8, cfg=_format(bits))
    said = L.paged_attention(b.Q, b.cache, b.pages, b.step, cfg=b.cfg)
    b.check(said)
    assert torch.equal(L.paged_attention(b.Q, b.cache, b.pages, b.step), said)
    for other in (3, 5, 7):
        with pytest.raises(ValueError, match="format"):
            L.paged_attention(b.Q, b.cache, b.pages, b.step, cfg=_format(other))


def test_a_cache_is_written_in_one_format():
    x = torch.randn((3, 2, 64), device=DEV)
    slots = torch.tensor([0, 5, 17], dtype=torch.int32, device=DEV)
    cache = L.new_kv_cache(2, 16, 2, 64, dtype=L.MXINT8, device=DEV)
    L.append_kv(x, x, cache, slots, cfg=_format(6))
    want = cache.keys.clone()
    cache.keys.zero_()
    L.append_kv(x, x, cache, slots)                        # in the cache's own
    assert torch.equal(cache.keys, want)
    with pytest.raises(ValueError, match="format"):
        L.append_kv(x, x, cache, slots, cfg=_format(8))
    assert torch.equal(cache.keys, want)


def test_the_format_may_be_given_with_the_cache():
    x = torch.randn((3, 2, 64), device=DEV)
    slots = torch.tensor([0, 5, 17], dtype=torch.int32, device=DEV)
    caches = [L.new_kv_cache(2, 16, 2, 64, dtype=L.MXINT8, device=DEV, cfg=c) for c in (_format(6), None)]
    L.append_kv(x, x, caches[0], slots)
    L.append_kv(x, x, caches[1], slots, cfg=_format(6))
    assert torch.equal(caches[0].keys, caches[1].keys) and torch.equal(caches[0].values, caches[1].values)
    with pytest.raises(ValueError, match="format"):
        L.append_kv(x, x, caches[0], slots, cfg=L.default_config())


def test_a_bf16_cache_has_none():
    b = Batch([(90, 2)], 8, 4, 128, 16)
    want = L.paged_attention(b.Q, b.cache, b.pages, b.step)
    assert torch.equal(L.paged_attention(b.Q, b.cache, b.pages, b.step, cfg=_format(6)), want)
    x = torch.randn((3, 4, 128), device=DEV)
    for bits in (6, 8):
        L.append_kv(x, x, b.cache, torch.tensor([0, 1, 2], dtype=torch.int32, device=DEV), cfg=_format(bits))
