"""Between the layers, at the far ends of what the calls take: tensors of more than 2^31 elements, the widest and the narrowest rows, the longest
contraction.  Rows from the front, from both sides of the 2^31st element and from the back are checked against 64 bits (bounds as in
test_gpu_boundary.py; adapters on whole numbers, exactly)."""
import numpy as np
import pytest
import torch

import paper_2402_02446_b200 as L
from oracle import mxint

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24


@pytest.fixture(autouse=True)
def _give_memory_back():
    yield
    torch.cuda.empty_cache()


def _some_rows(M, N):
    at = 2 ** 31 // N
    rows = sorted({0, 1, min(at - 1, M - 1), min(at, M - 1), min(at + 1, M - 1), min(2 * at, M - 1), M - 2, M - 1})
    return torch.tensor([r for r in rows if r >= 0], device=DEV)


def _randn(shape, seed, dtype):
    g = torch.Generator(device=DEV).manual_seed(seed)
    t = torch.empty(shape, dtype=dtype, device=DEV)
    for part in t.split(max(1, 2 ** 28 // shape[-1])):
        part.copy_(torch.randn(part.shape, generator=g, device=DEV))
    return t


def _check(Y, M, N, rows, want, rel):
    """Y: bf16 or fp32 [M, N], or MXINT8; want: fp64 of some rows."""
    if Y.dtype != torch.uint8:
        got, half = Y[rows].double(), 2.0 ** -8 if Y.dtype == torch.bfloat16 else 0.0
        assert bool(((got - want).abs() <= want.abs() * (rel + half * (1 + rel)) + 2.0 ** -102).all())
        return
    m, e = mxint.quantize(want.cpu().numpy(), 8, 1)
    Ym, Ye = L.split_mxint8(Y, M, N)
    assert np.array_equal(Ym[rows].cpu().numpy(), m) and np.array_equal(Ye[rows].cpu().numpy(), mxint.exponent_bytes(e))


SIZES = [(140000, 16384), (5, 2 ** 20), (3, 8), (100001, 16)]


@pytest.mark.parametrize("M,K", SIZES)
def test_norm(M, K):
    X, res, w = _randn((M, K), 1, torch.bfloat16), _randn((M, K), 2, torch.bfloat16), 1 + 0.2 * _randn((K,), 3, torch.float32)
    rows = _some_rows(M, K)
    h = (X[rows].float() + res[rows].float()).bfloat16().double()
    want = h / torch.sqrt((h * h).mean(1, keepdim=True) + 1e-5) * w.double()
    for dt in (torch.bfloat16,) + ((L.MXINT8,) if K % 16 == 0 else ()):
        own = res.clone()
        Y, _ = L.add_rms_norm(X, w, 1e-5, residual=own, residual_out=own, out_dtype=dt)
        assert torch.equal(own[rows].double(), h)
        _check(Y, M, K, rows, want, 4 * U)
        del own, Y


@pytest.mark.parametrize("M,N", SIZES + [(3, 2 ** 22)])
def test_gate_and_values(M, N):
    both = _randn((M, 2 * N), 4, torch.bfloat16)
    gate, up = both[:, :N], both[:, N:]
    rows = _some_rows(M, N)
    g = gate[rows].double()
    want = g / (1 + torch.exp(-g)) * up[rows].double()
    _check(L.gated_activation(gate, up, out_dtype=torch.bfloat16), M, N, rows, want, 12 * U)
    if N % 16 == 0:
        Y = L.gated_activation(gate, up)
        _check(Y, M, N, rows, want, 0)
        if N <= 2 ** 20:
            m, e = L.split_mxint8(Y, M, N)
            back = L.dequantize_activations(Y, M, N, out_dtype=torch.bfloat16)
            values = m[rows].double() * torch.exp2(e[rows].double() - 133).repeat_interleave(16, 1)
            assert torch.equal(back[rows].double(), values)


@pytest.mark.parametrize("M,K,N,rank,x,y", [(300000, 64, 8192, 16, "bf16", "bf16"), (300000, 64, 8192, 16, "bf16", "f32"), (262200, 8208, 16, 8, "mxint8", "f32"),
                                            (140000, 16400, 8, 40, "bf16", "bf16"), (1000, 48, 2 ** 22, 16, "bf16", "bf16"), (3, 2 ** 20, 8, 16, "f32", "f32"),
                                            (2, 16, 2 ** 22, 256, "bf16", "f32"), (1030, 2 ** 20, 8, 5, "mxint8", "f32")])
def test_adapters(M, K, N, rank, x, y):
    def whole(shape, seed, dtype, keep=1.0):
        g = torch.Generator(device=DEV).manual_seed(seed)
        t = torch.empty(shape, dtype=dtype, device=DEV)
        for part in t.split(max(1, 2 ** 28 // shape[-1])):
            part.copy_(torch.randint(-1, 2, part.shape, generator=g, device=DEV, dtype=torch.int8))
            if keep < 1:
                part.mul_(torch.rand(part.shape, generator=g, device=DEV) < keep)
        return t
    types = {"f32": torch.float32, "bf16": torch.bfloat16}
    X = whole((M, K), 5, torch.int8 if x == "mxint8" else types[x])
    # few enough of each column that T stays below 2^8 and the sums below 2^16: exact in bf16 parts and in fp32
    A, B = whole((K, rank), 6, torch.bfloat16, min(1.0, 40.0 / K)), whole((rank, N), 7, torch.bfloat16)
    pool = L.new_adapter_pool(K, N, rank, 3)
    L.load_adapter(pool, 1, A, B, 1.0)
    slots = torch.ones(M, dtype=torch.int32, device=DEV)
    slots[M // 3: M // 3 + M // 5] = -1
    Y0 = torch.empty((M, N), dtype=types[y], device=DEV)
    Y0.copy_((torch.arange(N, device=DEV) % 5)[None])
    Xt = X if x != "mxint8" else L.to_mxint8(X, torch.full((M, K // 16), 133, dtype=torch.uint8, device=DEV))
    plan = L.adapter_plan(slots, pool)
    Y = L.apply_adapters(Xt, pool, plan, Y0, Y=Y0)
    assert L.poll_status(plan.buf) == 0
    rows = torch.cat([_some_rows(M, N), _some_rows(M, K), torch.tensor([M // 3, M // 2], device=DEV)])
    T = X[rows].double() @ A.double()
    assert T.abs().max() < 256
    term = T @ B.double()
    term[slots[rows] < 0] = 0
    want = term + (torch.arange(N, device=DEV) % 5).double()
    assert torch.equal(Y[rows], want.to(types[y]))
