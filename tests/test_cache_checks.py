"""Host-side argument checks of the cache of keys and values and of the attention over it: refused before anything is launched, without a device."""
import ctypes as C

import pytest
import torch

import paper_2402_02446_b200 as L
from paper_2402_02446_b200 import binding

E = binding.STATUS_NAMES.index
F32, BF16, MX = 0, 1, 2
P = 4096                       # an aligned address that is never read


def _cache(k=P, v=2 * P, n_pages=8, page=16, heads=2, dim=64, dtype=BF16):
    return C.byref(binding._Cache(k, v, n_pages, page, heads, dim, dtype))


def _table(t=P, f=2 * P, R=4, max_pages=4, n_pages=8, page=16):
    return C.byref(binding._Table(t, f, R, max_pages, n_pages, page))


def _bad_cfg():
    bad = L.default_config()
    bad.a_bits = 9
    return C.byref(bad)


BAD_CACHES = [dict(n_pages=0), dict(n_pages=1 << 27), dict(page=0), dict(page=8), dict(page=48), dict(page=256), dict(heads=0), dict(heads=1025),
              dict(dim=96), dict(dim=0), dict(dim=256)]
BAD_TABLES = [dict(R=0), dict(R=16385), dict(max_pages=0), dict(max_pages=(1 << 26) + 1), dict(R=16384, max_pages=1 << 17), dict(n_pages=0),
              dict(n_pages=1 << 27), dict(page=17)]


def test_sizes():
    out = C.c_size_t()
    size = L.lib().lqer_kv_cache_bytes
    assert size(_cache(), C.byref(out)) == 0 and out.value == 8 * 2 * 16 * 64 * 2
    assert size(_cache(dtype=MX), C.byref(out)) == 0 and out.value == 8 * 2 * 16 * 68
    assert size(None, C.byref(out)) == size(_cache(), None) == E("LQER_ERR_NULL")
    assert size(_cache(dtype=F32), C.byref(out)) == size(_cache(dtype=7), C.byref(out)) == E("LQER_ERR_CONFIG")
    for kw in BAD_CACHES:
        assert size(_cache(**kw), C.byref(out)) == E("LQER_ERR_SHAPE"), kw
    step = L.lib().lqer_cache_step_bytes
    assert step(4, C.byref(out)) == 0 and out.value >= 256 + 64
    assert step(0, C.byref(out)) == step(16385, C.byref(out)) == E("LQER_ERR_SHAPE")
    assert step(4, None) == E("LQER_ERR_NULL")


def test_step_refusals():
    def step(table=None, le=3 * P, added=4 * P, ring=5 * P, M=8, most=8, lo=6 * P, ro=7 * P, slots=8 * P, pos=9 * P, plan=10 * P, size=1 << 20, **kw):
        return L.lib().lqer_cache_step(_table(**kw) if table is None else table, le, added, ring, M, most, lo, ro, slots, pos, plan, size, None)

    for kw in (dict(le=None), dict(added=None), dict(ring=None), dict(lo=None), dict(ro=None), dict(slots=None), dict(pos=None), dict(plan=None), dict(t=None),
               dict(f=None), dict(table=C.POINTER(binding._Table)())):
        assert step(**kw) == E("LQER_ERR_NULL"), kw
    for kw in BAD_TABLES + [dict(M=0), dict(M=-1), dict(M=(1 << 24) + 1), dict(most=0)]:
        assert step(**kw) == E("LQER_ERR_SHAPE"), kw
    for kw in (dict(t=P + 2), dict(f=P + 1), dict(le=P + 2), dict(added=P + 1), dict(ring=P + 4), dict(ro=P + 4), dict(slots=P + 2), dict(pos=P + 3), dict(plan=P + 16)):
        assert step(**kw) == E("LQER_ERR_ALIGN"), kw
    assert step(size=256) == E("LQER_ERR_BUFFER_TOO_SMALL")
    for kw in (dict(lo=4 * P), dict(pos=8 * P), dict(f=P)):
        assert step(**kw) == E("LQER_ERR_CONFIG"), kw


def test_append_refusals():
    def append(K=3 * P, V=4 * P, xt=F32, ks=128, vs=128, M=4, slots=5 * P, cache=None, cfg=None, **kw):
        return L.lib().lqer_append_kv(K, V, xt, ks, vs, M, slots, _cache(**kw) if cache is None else cache, cfg, None)

    for kw in (dict(K=None), dict(V=None), dict(slots=None), dict(k=None), dict(v=None), dict(cache=C.POINTER(binding._Cache)())):
        assert append(**kw) == E("LQER_ERR_NULL"), kw
    for kw in BAD_CACHES + [dict(M=0), dict(M=(1 << 24) + 1), dict(ks=120), dict(vs=0), dict(ks=132), dict(vs=129), dict(ks=(1 << 32) + 8)]:
        assert append(**kw) == E("LQER_ERR_SHAPE"), kw
    for kw in (dict(K=P + 8), dict(V=P + 8), dict(slots=P + 2), dict(k=P + 8), dict(v=P + 8)):
        assert append(**kw) == E("LQER_ERR_ALIGN"), kw
    for kw in (dict(xt=MX), dict(xt=-1), dict(v=P), dict(cfg=_bad_cfg()), dict(dtype=F32)):
        assert append(**kw) == E("LQER_ERR_CONFIG"), kw


def test_attention_refusals():
    size = C.c_size_t()
    need = L.lib().lqer_attention_workspace_bytes

    def attend(Q=3 * P, stride=256, M=4, heads=4, cache=None, table=None, step=4 * P, most=1, window=0, sinks=0, scale=1.0, cfg=None, Y=5 * P, ws=6 * P,
               room=1 << 40, **kw):
        of_cache = {k: v for k, v in kw.items() if k in ("k", "v", "n_pages", "page", "heads_kv", "dim", "dtype")}
        if "heads_kv" in of_cache:
            of_cache["heads"] = of_cache.pop("heads_kv")
        of_table = {k: v for k, v in kw.items() if k in ("t", "f", "R", "max_pages", "table_pages", "table_page")}
        for a, b in (("table_pages", "n_pages"), ("table_page", "page")):
            if a in of_table:
                of_table[b] = of_table.pop(a)
        return L.lib().lqer_paged_attention(Q, stride, M, heads, _cache(**of_cache) if cache is None else cache, _table(**of_table) if table is None else table,
                                            step, most, window, sinks, scale, cfg, Y, ws, room, None)

    for kw in (dict(Q=None), dict(Y=None), dict(step=None), dict(k=None), dict(v=None), dict(t=None), dict(ws=None), dict(cache=C.POINTER(binding._Cache)()),
               dict(table=C.POINTER(binding._Table)())):
        assert attend(**kw) == E("LQER_ERR_NULL"), kw
    for kw in (dict(M=0), dict(M=(1 << 24) + 1), dict(heads=0), dict(heads=3), dict(heads=1026, stride=1 << 17), dict(M=1 << 24, heads=128, stride=1 << 14), dict(most=0), dict(stride=248), dict(stride=260),
               dict(stride=(1 << 32) + 8), dict(window=-1), dict(sinks=-1), dict(page=8), dict(dim=96), dict(heads_kv=0), dict(R=0), dict(max_pages=0),
               dict(table_pages=9), dict(table_page=32)):
        assert attend(**kw) == E("LQER_ERR_SHAPE"), kw
    for kw in (dict(Q=P + 8), dict(Y=P + 8), dict(step=P + 16), dict(ws=P + 16), dict(k=P + 8), dict(t=P + 2)):
        assert attend(**kw) == E("LQER_ERR_ALIGN"), kw
    for kw in (dict(Y=3 * P), dict(Y=P), dict(Y=2 * P), dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=-1e30), dict(dtype=F32), dict(cfg=_bad_cfg())):
        assert attend(**kw) == E("LQER_ERR_CONFIG"), kw
    assert need(4, 4, _cache(), _table(), 1, None) == E("LQER_ERR_NULL")
    assert need(4, 4, None, _table(), 1, C.byref(size)) == need(4, 4, _cache(), None, 1, C.byref(size)) == E("LQER_ERR_NULL")
    assert need(4, 3, _cache(), _table(), 1, C.byref(size)) == need(0, 4, _cache(), _table(), 1, C.byref(size)) == E("LQER_ERR_SHAPE")


def test_the_binding_looks_at_its_tensors():
    cpu = torch.zeros(4, dtype=torch.int32)
    pages = L.new_page_table(4, 4, 8, 16, device="cpu")
    cache = L.new_kv_cache(8, 16, 2, 64, device="cpu")
    assert cache.keys.shape == (8, 2, 16, 64) and pages.tables.shape == (4, 4) and pages.ring.tolist() == [0, 8]
    for bad in (lambda: L.cache_step(pages, cpu, 4), lambda: L.append_kv(torch.zeros(4, 2, 64), torch.zeros(4, 2, 64), cache, cpu),
                lambda: L.paged_attention(torch.zeros((4, 4, 64), dtype=torch.bfloat16), cache, pages, None),
                lambda: L.new_kv_cache(8, 16, 2, 64, dtype=torch.float32, device="cpu")):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(L.LqerError):
        L.new_kv_cache(8, 16, 2, 96, device="cpu")
    with pytest.raises(L.LqerError):
        L.new_page_table(0, 4, 8, 16, device="cpu")
    assert L.launch_count() == 0
