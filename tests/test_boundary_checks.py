"""Host-side argument checks of what stands between the layers: refused before anything is launched, without a device."""
import ctypes as C

import pytest
import torch

import paper_2402_02446_b200 as L
from paper_2402_02446_b200 import binding

E = binding.STATUS_NAMES.index
F32, BF16, MX = 0, 1, 2
P = 4096                       # an aligned address that is never read


def _norm(X=P, xt=F32, res=2 * P, out=2 * P, rt=F32, w=3 * P, wt=F32, eps=1e-5, M=4, K=64, cfg=None, Y=5 * P, yt=F32):
    return L.lib().lqer_add_rms_norm(X, xt, res, out, rt, w, wt, eps, M, K, cfg, Y, yt, None)


def test_norm_refusals():
    for kw in (dict(X=None), dict(w=None), dict(Y=None)):
        assert _norm(**kw) == E("LQER_ERR_NULL")
    for kw in (dict(M=0), dict(M=-1), dict(M=(1 << 24) + 1), dict(K=0), dict(K=60), dict(K=72, yt=MX), dict(K=(1 << 20) + 16)):
        assert _norm(**kw) == E("LQER_ERR_SHAPE"), kw
    for kw in (dict(X=P + 4), dict(res=P + 8), dict(out=P + 8), dict(w=P + 2), dict(Y=P + 8)):
        assert _norm(**kw) == E("LQER_ERR_ALIGN"), kw
    for kw in (dict(xt=MX), dict(rt=MX), dict(wt=MX), dict(yt=3), dict(xt=-1), dict(eps=-1.0), dict(eps=float("nan")), dict(Y=P), dict(Y=2 * P),
               dict(out=P, rt=BF16)):
        assert _norm(**kw) == E("LQER_ERR_CONFIG"), kw
    bad = L.default_config()
    bad.a_bits = 9
    assert _norm(cfg=C.byref(bad)) == E("LQER_ERR_CONFIG")


def test_gate_and_dequantize_refusals():
    def gate(g=P, u=2 * P, xt=F32, ld=64, M=4, N=64, act=0, cfg=None, Y=5 * P, yt=F32):
        return L.lib().lqer_gated_activation(g, u, xt, ld, M, N, act, cfg, Y, yt, None)

    for kw in (dict(g=None), dict(u=None), dict(Y=None)):
        assert gate(**kw) == E("LQER_ERR_NULL")
    for kw in (dict(M=0), dict(N=0), dict(N=60), dict(N=56, yt=MX, ld=56), dict(ld=56), dict(ld=68), dict(N=(1 << 22) + 8, ld=1 << 23)):
        assert gate(**kw) == E("LQER_ERR_SHAPE"), kw
    for kw in (dict(g=P + 8), dict(u=P + 8), dict(Y=P + 8)):
        assert gate(**kw) == E("LQER_ERR_ALIGN"), kw
    for kw in (dict(xt=MX), dict(act=2), dict(act=-1), dict(yt=5), dict(Y=P), dict(Y=2 * P)):
        assert gate(**kw) == E("LQER_ERR_CONFIG"), kw

    def back(X=P, M=4, K=64, Y=5 * P, yt=F32):
        return L.lib().lqer_dequantize_activations(X, M, K, None, Y, yt, None)

    assert back(X=None) == back(Y=None) == E("LQER_ERR_NULL")
    assert back(M=0) == back(K=72) == back(K=0) == E("LQER_ERR_SHAPE")
    assert back(X=P + 8) == back(Y=P + 8) == E("LQER_ERR_ALIGN")
    assert back(yt=MX) == back(Y=P) == E("LQER_ERR_CONFIG")


def _pool(data=P, K=64, N=64, max_rank=16, n_slots=4):
    return C.byref(binding._Pool(data, K, N, max_rank, n_slots))


def test_adapter_refusals():
    lib, size = L.lib(), C.c_size_t()
    assert lib.lqer_adapter_pool_bytes(None, C.byref(size)) == lib.lqer_adapter_pool_bytes(_pool(), None) == E("LQER_ERR_NULL")
    bad_shapes = (dict(K=60), dict(K=0), dict(N=60), dict(N=0), dict(max_rank=0), dict(max_rank=257), dict(n_slots=0), dict(n_slots=1025))
    for kw in bad_shapes:
        assert lib.lqer_adapter_pool_bytes(_pool(**kw), C.byref(size)) == E("LQER_ERR_SHAPE"), kw
    assert lib.lqer_adapter_pool_bytes(_pool(None), C.byref(size)) == 0            # the size needs no memory
    # a head, and 2 bytes an entry: A by blocks of 64 rows and 16 ranks, B by blocks of 128 columns and 16, 32 or 64 ranks
    assert size.value == 4 * (256 + 2 * 64 * 16 + 2 * 128 * 16)
    assert lib.lqer_adapter_pool_init(_pool(), size.value - 1, None) == E("LQER_ERR_BUFFER_TOO_SMALL")
    assert lib.lqer_adapter_pool_init(_pool(None), size.value, None) == E("LQER_ERR_NULL")
    assert lib.lqer_adapter_pool_init(_pool(P + 16), size.value, None) == E("LQER_ERR_ALIGN")

    def load(pool=_pool(), slot=0, A=P, B=P, dt=F32, rank=4):
        return lib.lqer_adapter_load(pool, slot, A, B, dt, rank, 1.0, None)

    assert load(A=None) == load(B=None) == E("LQER_ERR_NULL")
    assert load(slot=-1) == load(slot=4) == load(rank=-1) == load(rank=17) == E("LQER_ERR_SHAPE")
    assert load(A=P + 4) == load(B=P + 4) == E("LQER_ERR_ALIGN")
    assert load(dt=MX) == E("LQER_ERR_CONFIG")

    assert lib.lqer_adapter_plan_bytes(0, 4, C.byref(size)) == lib.lqer_adapter_plan_bytes(4, 1025, C.byref(size)) == E("LQER_ERR_SHAPE")
    assert lib.lqer_adapter_plan_bytes(4, 4, None) == E("LQER_ERR_NULL")
    assert lib.lqer_adapter_plan_bytes(33, 4, C.byref(size)) == 0
    need = size.value

    def plan(slots=P, M=33, n=4, buf=P, nbytes=need):
        return lib.lqer_adapter_plan(slots, M, n, buf, nbytes, None)

    assert plan(slots=None) == plan(buf=None) == E("LQER_ERR_NULL")
    assert plan(M=0) == plan(n=0) == E("LQER_ERR_SHAPE")
    assert plan(slots=P + 2) == plan(buf=P + 128) == E("LQER_ERR_ALIGN")
    assert plan(nbytes=need - 1) == E("LQER_ERR_BUFFER_TOO_SMALL")

    def apply(X=P, xt=F32, M=4, pool=_pool(), buf=P, n=4, Y0=2 * P, y0t=F32, Y=3 * P, yt=F32, cfg=None, ws=None, nbytes=0):
        return lib.lqer_adapters(X, xt, M, pool, buf, n, Y0, y0t, Y, yt, cfg, ws, nbytes, None)

    for kw in (dict(X=None), dict(pool=None), dict(buf=None), dict(Y0=None), dict(Y=None), dict(pool=_pool(None))):
        assert apply(**kw) == E("LQER_ERR_NULL"), kw
    for kw in (dict(M=0), dict(n=5), dict(n=0), *(dict(pool=_pool(**s)) for s in bad_shapes)):
        assert apply(**kw) == E("LQER_ERR_SHAPE"), kw
    for kw in (dict(X=P + 8), dict(Y0=P + 8), dict(Y=P + 8), dict(buf=P + 16), dict(pool=_pool(P + 16))):
        assert apply(**kw) == E("LQER_ERR_ALIGN"), kw
    for kw in (dict(xt=3), dict(y0t=MX), dict(yt=MX), dict(Y=P), dict(Y=2 * P, yt=BF16)):
        assert apply(**kw) == E("LQER_ERR_CONFIG"), kw
    # more than 512 rows go through a workspace
    assert lib.lqer_adapters_workspace_bytes(512, _pool(), 4, C.byref(size)) == 0 and size.value == 0
    assert lib.lqer_adapters_workspace_bytes(1024, _pool(), 4, C.byref(size)) == 0 and size.value == 0      # a small product
    big = dict(K=4096, N=11008, max_rank=64)
    assert lib.lqer_adapters_workspace_bytes(640, _pool(**big), 4, C.byref(size)) == 0 and size.value > 0
    assert lib.lqer_adapters_workspace_bytes(1025, _pool(), 4, C.byref(size)) == 0 and size.value > 0
    assert lib.lqer_adapters_workspace_bytes(513, _pool(), 5, C.byref(size)) == lib.lqer_adapters_workspace_bytes(0, _pool(), 4, C.byref(size)) == E("LQER_ERR_SHAPE")
    assert lib.lqer_adapters_workspace_bytes(513, _pool(), 4, None) == E("LQER_ERR_NULL")
    assert apply(M=1025) == E("LQER_ERR_NULL") and apply(M=1025, ws=P + 16, nbytes=1 << 30) == E("LQER_ERR_ALIGN")
    assert apply(M=1025, ws=P, nbytes=size.value - 1) == E("LQER_ERR_BUFFER_TOO_SMALL")
    assert L.launch_count() == 0


def test_tensors_on_the_host_are_refused():
    x, w = torch.zeros((2, 64)), torch.ones(64)
    for call in (lambda: L.add_rms_norm(x, w, 1e-5), lambda: L.gated_activation(x, x), lambda: L.dequantize_activations(torch.zeros(136, dtype=torch.uint8), 2, 64),
                 lambda: L.add_rms_norm(x, w[:32], 1e-5), lambda: L.add_rms_norm(x[0], w, 1e-5), lambda: L.gated_activation(x, w),
                 lambda: L.gated_activation(x[:, ::2], x[:, ::2])):
        with pytest.raises(ValueError):
            call()


def test_a_plan_has_room_for_every_batch():
    # the head, slot and length (8 bytes) of every tile that any batch can have, its rows: tiles of 8 up to 1024 rows, of 128 above 512
    size = C.c_size_t()
    for M in (1, 2, 7, 8, 9, 15, 16, 17, 100, 512, 513, 1024, 1025, 4096):
        for n in (1, 2, 7, 64, 1024):
            assert L.lib().lqer_adapter_plan_bytes(M, n, C.byref(size)) == 0
            need = 256
            for rows in ([8] if M <= 1024 else []) + ([128] if M > 512 else []):
                # the worst batch: as many bins as possible with one row more than a whole number of tiles
                bins = min(n + 1, M)
                worst = sum(-(-r // rows) for r in [1] * (bins - 1) + [M - (bins - 1)])
                need += 8 * worst + 4 * rows * worst
            assert size.value >= need, (M, n)


def test_a_result_has_its_own_shape_whatever_its_inputs():
    # an MXINT8 buffer may come in two dimensions: what is made beside it is [M, K] all the same
    for shape in ((4, 68), (1, 272), (272,), (2, 136)):
        for dt in (torch.float32, torch.bfloat16):
            Y, _, _ = binding._output(None, 4, 64, dt, torch.zeros(shape, dtype=torch.uint8), -1)
            assert Y.shape == (4, 64) and Y.dtype == dt and Y.is_contiguous()
    Y, _, _ = binding._output(None, 4, 64, torch.bfloat16, torch.zeros((4, 128))[:, :64], -1)
    assert Y.shape == (4, 64) and Y.is_contiguous()
