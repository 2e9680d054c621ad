"""Between the layers: the norm with the residual's addition, the gated activation and MXINT8 read back as values, against
64-bit arithmetic.

Bounds (u = 2^-24, half a step of fp32).  Norm: the inverse root, its product with h and the product with the weight are rounded
once each: 3 u.  Gate: expf 4 u, the sum u, the quotient 4 u, the product u, so 10 u, and what seven roundings of z do to exp(z), 7 u |z|
(GELU; SiLU's argument is exact).  bf16 results add half a bf16 step (2^-8), MXINT8 results are those of 64-bit values exactly.
"""
import math

import numpy as np
import pytest
import torch

import paper_2402_02446_b200 as L
from oracle import mxint
from paper_2402_02446_b200 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _cfg(bits=8, lo=-56, hi=55):
    cfg = L.default_config()
    cfg.a_bits, cfg.exp_min, cfg.exp_max = bits, lo, hi
    return cfg


def _values(shape, seed, dtype, spread=6):
    """Values over a dozen binades, with some zeros."""
    g = torch.Generator().manual_seed(seed)
    v = torch.randn(shape, generator=g) * torch.exp2(torch.randint(-spread, spread + 1, shape, generator=g).float())
    v[torch.rand(shape, generator=g) < 0.02] = 0.0
    return v.to(dtype).to(DEV)


def _check(Y, want, rel, M, N, kind, cfg, tiny=2.0 ** -126):
    """want: fp64 numpy values; rel: bound on the fp32 result's relative error, beside `tiny`."""
    if kind == "mxint8":
        m, e = mxint.quantize(want, cfg.a_bits, 1, exp_min=cfg.exp_min, exp_max=cfg.exp_max)
        Ym, Ye = L.split_mxint8(Y, M, N)
        assert np.array_equal(Ye.cpu().numpy(), mxint.exponent_bytes(e))
        assert np.array_equal(Ym.cpu().numpy(), m)
        for dt in (torch.float32, torch.bfloat16):
            back = L.dequantize_activations(Y, M, N, out_dtype=dt, cfg=cfg)
            assert back.dtype == dt and np.array_equal(back.double().cpu().numpy(), mxint.dequantize(m, e, cfg.a_bits, 1))
        return
    assert Y.dtype == TYPES[kind]
    got = Y.double().cpu().numpy()
    bound = np.abs(want) * (rel + (2.0 ** -8 if kind == "bf16" else 0.0) * (1 + rel)) + tiny
    assert np.all(np.abs(got - want) <= bound), float(np.max(np.abs(got - want) / bound))


def _norm64(h, w, eps):
    h, w = h.double().cpu().numpy(), w.double().cpu().numpy()
    return h * (1.0 / np.sqrt((h * h).sum(1, keepdims=True) / h.shape[1] + eps)) * w


@pytest.mark.parametrize("y", ["f32", "bf16", "mxint8"])
@pytest.mark.parametrize("r", ["f32", "bf16"])
@pytest.mark.parametrize("x", ["f32", "bf16"])
@pytest.mark.parametrize("M,K", [(1, 16), (3, 256), (1, 4096), (5, 4112), (2, 8208), (201, 272), (3, 16400), (2, 32784)])
def test_add_rms_norm(M, K, x, r, y):
    X, res = _values((M, K), 1, TYPES[x]), _values((M, K), 2, TYPES[r])
    w = 1.0 + 0.2 * _values((K,), 3, torch.float32, 0)
    cfg = _cfg(6 if K == 272 else 8)
    h = (X.float() + res.float()).to(TYPES[r])
    Y, out = L.add_rms_norm(X, w, 1e-5, residual=res, out_dtype=L.MXINT8 if y == "mxint8" else TYPES[y], cfg=cfg)
    assert out.dtype == res.dtype and torch.equal(out, h)
    _check(Y, _norm64(h, w, 1e-5), 3 * U * (1 + 4 * U), M, K, y, cfg)


def test_add_rms_norm_many_rows_at_the_borders():
    # 4 M elements, so that some lie next to every kind of border; small integers make exact powers of two and equal squares
    M, K = 1024, 4096
    X = _values((M, K), 5, torch.bfloat16, 1)
    X[: M // 2] = torch.randint(-3, 4, (M // 2, K), generator=torch.Generator().manual_seed(6)).to(torch.bfloat16).to(DEV)
    w = torch.ones(K, device=DEV)
    Y, _ = L.add_rms_norm(X, w, 0.0)
    _check(Y, _norm64(X, w, 0.0), 0, M, K, "mxint8", _cfg())


def test_add_rms_norm_forms():
    M, K = 7, 1040
    X, res, w = _values((M, K), 7, torch.float32), _values((M, K), 8, torch.float32), _values((K,), 9, torch.bfloat16, 0)
    want = _norm64(X + res, w, 1e-6)
    # residual in place, and the result's buffer given
    r2, Y = res.clone(), torch.full((M, K), 7.0, device=DEV)
    got, out = L.add_rms_norm(X, w, 1e-6, residual=r2, residual_out=r2, Y=Y)
    assert got is Y and out is r2 and torch.equal(r2, X + res)
    _check(Y, want, 3 * U * (1 + 4 * U), M, K, "f32", None)
    # X's buffer takes the sum
    x2 = X.clone()
    got, out = L.add_rms_norm(x2, w, 1e-6, residual=res, residual_out=x2, out_dtype=torch.float32)
    assert torch.equal(x2, X + res) and torch.equal(got, Y)
    # no residual: h is X, kept or not
    got, out = L.add_rms_norm(X, w, 1e-6, out_dtype=torch.float32)
    assert out is None
    _check(got, _norm64(X, w, 1e-6), 3 * U * (1 + 4 * U), M, K, "f32", None)
    b = torch.empty((M, K), dtype=torch.bfloat16, device=DEV)
    got, out = L.add_rms_norm(X, w, 1e-6, residual_out=b, out_dtype=torch.float32)
    assert out is b and torch.equal(b, X.bfloat16())
    _check(got, _norm64(b, w, 1e-6), 3 * U * (1 + 4 * U), M, K, "f32", None)


@pytest.mark.parametrize("K", [64, 33024])
def test_add_rms_norm_in_place_over_a_long_row(K):
    # the residual's buffer is an input and an output: the sum goes in once, also where a row is read twice
    X, res, w = _values((2, K), 10, torch.float32), _values((2, K), 11, torch.float32), torch.ones(K, device=DEV)
    h = X + res
    Y, out = L.add_rms_norm(X, w, 1e-5, residual=res, residual_out=res)
    assert torch.equal(out, h) and out is res
    _check(Y, _norm64(h, w, 1e-5), 0, 2, K, "mxint8", _cfg())


def test_add_rms_norm_special_values():
    K = 256
    X = torch.ones((6, K), device=DEV)
    X[0, 5] = float("nan")
    X[1, 7] = float("inf")
    X[2] = 0.0
    X[3] *= 1e30                 # squares beyond fp32
    X[4] *= 3e38
    w = torch.ones(K, device=DEV)
    Y, _ = L.add_rms_norm(X, w, 0.0, out_dtype=torch.float32)
    assert torch.isnan(Y[0]).all() and torch.isnan(Y[1, 7]) and (Y[1, :7] == 0).all() and torch.isnan(Y[2]).all()
    assert torch.allclose(Y[3:6], torch.ones((3, K), device=DEV), rtol=1e-6)
    m, e = L.split_mxint8(L.add_rms_norm(X, w, 0.0)[0], 6, K)
    assert (m[0] == 0).all() and (e[0] == 127 - 56).all() and (m[1] == 0).all() and (m[2] == 0).all()
    assert (m[3:6] == 64).all() and (e[3:6] == 127).all()
    # an eps keeps a zero row zero
    Y, _ = L.add_rms_norm(X[2:3].contiguous(), w, 1e-5, out_dtype=torch.float32)
    assert (Y == 0).all()


@pytest.mark.parametrize("K", [256, 4096, 4112, 8208, 16400, 33024])
@pytest.mark.parametrize("x", ["f32", "bf16"])
def test_add_rms_norm_rows_that_lie_on_a_border(x, K):
    # rows of one magnitude: h / rms is +-1, the lower border of an exponent, whatever the magnitude
    c = torch.arange(1, 128, device=DEV, dtype=torch.float32)[:, None]
    sign = torch.randint(0, 2, (127, K), generator=torch.Generator(device=DEV).manual_seed(71), device=DEV) * 2 - 1
    h = (c * sign).to(TYPES[x])
    res = (h.float() * 0.5 if x == "f32" else torch.zeros_like(h)).to(TYPES[x])
    w = torch.exp2(torch.arange(K, device=DEV).float() // 16 % 3)
    m, e = L.split_mxint8(L.add_rms_norm(h - res, w, 0.0, residual=res)[0], 127, K)
    assert (m == 64 * sign).all() and (e.int() - 127 == torch.arange(K // 16, device=DEV) % 3).all()
    # half of each row a, half 7 a: rms 5 a; 7 / 5 * 1.25 is a value with seven bits, 1 / 5 * 1.25 a power of two
    h = torch.where(torch.arange(K, device=DEV) % 2 == 0, c, 7 * c)
    h = h[(7 * c[:, 0]).to(TYPES[x]) == 7 * c[:, 0]].to(TYPES[x])
    m, e = L.split_mxint8(L.add_rms_norm(h, torch.full((K,), 1.25, device=DEV), 0.0)[0], h.shape[0], K)
    assert (m[:, 1::2] == 112).all() and (m[:, ::2] == 16).all() and (e == 127).all()


@pytest.mark.parametrize("K", [264, 4104, 8200, 16392, 33024])
@pytest.mark.parametrize("x", ["f32", "bf16"])
def test_add_rms_norm_rows_near_the_ends_of_the_range(x, K):
    # the inverse root of such rows is beyond fp32, or not a normal number there; their norms are ordinary numbers
    size = torch.tensor([1e-40, 4e-39, 1.3e-38, 1e-36, 1e-30, 1e30, 1e36, 2e37, 8e37, 1.6e38], dtype=torch.float64, device=DEV)
    X = (size[:, None] * (0.5 + 1.5 * torch.rand((len(size), K), generator=torch.Generator(device=DEV).manual_seed(72), device=DEV).double())).to(TYPES[x])
    w = 1.0 + 0.2 * _values((K,), 73, torch.float32, 0)
    want = _norm64(X, w, 0.0)
    for y in ("f32", "bf16"):
        Y, _ = L.add_rms_norm(X, w, 0.0, out_dtype=TYPES[y])
        _check(Y, want, 3 * U * (1 + 4 * U), len(size), K, y, None)


def _act64(g, act):
    with np.errstate(over="ignore"):
        z = g if act == "silu" else 2.0 * math.sqrt(2.0 / math.pi) * (g + 0.044715 * g ** 3)
        return g / (1.0 + np.exp(-z)), np.zeros_like(z) if act == "silu" else np.abs(z)


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("y", ["f32", "bf16", "mxint8"])
@pytest.mark.parametrize("x", ["f32", "bf16"])
@pytest.mark.parametrize("M,N,joined", [(1, 16, False), (3, 256, True), (1, 11008, True), (37, 1040, False), (200, 2064, True)])
def test_gated_activation(M, N, joined, x, y, act):
    if joined:
        both = _values((M, 2 * N), 21, TYPES[x], 3)
        gate, up = both[:, :N], both[:, N:]
    else:
        gate, up = _values((M, N), 21, TYPES[x], 3), _values((M, N), 22, TYPES[x])
    cfg = _cfg(6 if M == 37 else 8)
    Y = L.gated_activation(gate, up, act=act, out_dtype=L.MXINT8 if y == "mxint8" else TYPES[y], cfg=cfg)
    a, z = _act64(gate.double().cpu().numpy(), act)
    want = a * up.double().cpu().numpy()
    # beyond z = -87 exp(-z) nears the end of fp32's range, where the quotient may come out as zero: the result is then below
    # |g u| exp(-87) < 2^14 * 2^-125, or, times |u| < 2^9, below 2^-102
    _check(Y, want, (10 + 7 * z) * U * (1 + 1e-5), M, N, y, cfg, tiny=2.0 ** -102)


def test_gated_activation_odd_width_and_window():
    # N a multiple of 8 but not of 16 (no MXINT8), and a narrow exponent window: everything saturates or vanishes as the oracle says
    gate, up = _values((5, 1048), 31, torch.float32, 3), _values((5, 1048), 32, torch.float32)
    Y = L.gated_activation(gate, up, out_dtype=torch.float32)
    a, z = _act64(gate.double().cpu().numpy(), "silu")
    _check(Y, a * up.double().cpu().numpy(), 10 * U * (1 + 1e-5), 5, 1048, "f32", None)
    with pytest.raises(ValueError):
        L.gated_activation(gate, up)
    g, u = gate[:, :1040].contiguous(), up[:, :1040].contiguous()
    cfg = _cfg(8, -2, 1)
    _check(L.gated_activation(g, u, cfg=cfg), _act64(g.double().cpu().numpy(), "silu")[0] * u.double().cpu().numpy(), 0, 5, 1040, "mxint8", cfg)


def test_gated_activation_large_negative_gates_keep_their_borders():
    # blocks whose maximum is itself the tail of exp: the error of z counts |z| times there
    g = torch.linspace(-30.0, -1.0, 64 * 512, device=DEV).view(64, 512)
    u = _values((64, 512), 33, torch.float32, 0)
    for act in ("silu", "gelu"):
        cfg = _cfg()
        _check(L.gated_activation(g, u, act=act, cfg=cfg), _act64(g.double().cpu().numpy(), act)[0] * u.double().cpu().numpy(), 0, 64, 512, "mxint8", cfg)


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("x", ["f32", "bf16"])
def test_gated_activation_special_values(x, act):
    # masks of the type's lowest value, infinities and NaN, alone in a block, all over a row, and beside ordinary values
    N, rows, inf, nan = 272, 16, float("inf"), float("nan")
    g, u = _values((rows, N), 61, TYPES[x], 2), _values((rows, N), 62, TYPES[x], 2)
    low = torch.finfo(TYPES[x]).min
    g[0], u[0] = low, 0.0                        # a masked row
    g[1] = low
    g[2, 16:48], u[2, 16:48] = low, 0.0          # masked blocks
    g[3, ::2] = low
    g[4], g[5] = -inf, inf
    g[6, 5], g[7, 21], u[8, 40] = -inf, inf, inf
    g[9, 3], u[10, 4], g[11, 64:80] = nan, nan, nan
    g[12, 7], u[12, 7] = 0.0, -inf
    g[13], u[13, ::2] = -200.0, 0.0
    g[14], u[14] = -1000.0, 2.0 ** 20
    g[15, ::3] = -90.0
    with np.errstate(all="ignore"):
        g64, u64 = g.double().cpu().numpy(), u.double().cpu().numpy()
        z = g64 if act == "silu" else 2.0 * math.sqrt(2.0 / math.pi) * (g64 + 0.044715 * g64 ** 3)
        want = g64 / (1.0 + np.exp(-z)) * u64
        tail = np.where(np.isfinite(g64 * u64), np.abs(g64 * u64) * 2.0 ** -126, 0.0) + 2.0 ** -126      # what may come out as zero
    rel = (10 + 7 * 90) * U
    for cfg in (_cfg(), _cfg(6, -40, 3)):
        _check(L.gated_activation(g, u, act=act, cfg=cfg), want, 0, rows, N, "mxint8", cfg)
    for y in ("f32", "bf16"):
        got = L.gated_activation(g, u, act=act, out_dtype=TYPES[y]).double().cpu().numpy()
        assert np.array_equal(np.isnan(got), np.isnan(want))
        assert np.array_equal(np.isinf(got), np.isinf(want)) and np.array_equal(np.sign(got[np.isinf(got)]), np.sign(want[np.isinf(want)]))
        at = np.isfinite(want)
        bound = np.abs(want[at]) * (rel + (2.0 ** -8 if y == "bf16" else 0.0) * (1 + rel)) + tail[at]
        assert (np.abs(got[at] - want[at]) <= bound).all()


def test_values_of_a_buffer_in_two_dimensions():
    M, K = 4, 64
    Xq = L.to_mxint8(*L.quantize_activations(_values((M, K), 45, torch.float32)))
    for dt in (torch.float32, torch.bfloat16):
        want = L.dequantize_activations(Xq, M, K, out_dtype=dt)
        assert want.shape == (M, K)
        for shape in ((M, 17 * K // 16), (1, -1), (2, -1)):
            got = L.dequantize_activations(Xq.view(shape), M, K, out_dtype=dt)
            assert got.shape == (M, K) and torch.equal(got, want)


def test_values_into_a_tensor_aligned_to_16_bytes_only():
    X = _values((9, 272), 44, torch.float32)
    Xq = L.to_mxint8(*L.quantize_activations(X))
    for dt in (torch.float32, torch.bfloat16):
        n = 16 // torch.empty(0, dtype=dt).element_size()
        Y = torch.empty(9 * 272 + 2 * n, dtype=dt, device=DEV)[n:n + 9 * 272].view(9, 272)
        assert Y.data_ptr() % 32 == 16 and torch.equal(L.dequantize_activations(Xq, 9, 272, Y=Y), L.dequantize_activations(Xq, 9, 272, out_dtype=dt))


def test_the_layer_takes_the_norms_output_as_its_own():
    # MXINT8 from the norm into the layer equals the fp32 values of that tensor into the layer, bit for bit
    import lqer_inputs as gen
    spec = gen.LayerSpec("boundary", M=9, K=512, N=264, k=16, calib_rows=32, outlier_frac=0.01, outlier_scale=20.0, seed=77)
    A, B = gen.make_random_factors(spec)
    P = L.prepare_weights(*(torch.from_numpy(np.ascontiguousarray(v)).to(DEV) for v in (gen.make_weight(spec), A, B)))
    ws = L.new_workspace(9, P)
    X, w = _values((9, 512), 41, torch.bfloat16), torch.ones(512, device=DEV)
    Yq, _ = L.add_rms_norm(X, w, 1e-5)
    a = L.linear_ex(Yq, P, ws, M=9)
    b = L.linear_ex(L.dequantize_activations(Yq, 9, 512), P, ws)
    assert L.poll_status(ws) == 0 and torch.equal(a, b)
    P.release()


def test_streams_and_graphs():
    # on a stream of its own behind the work that makes the input, and replayed from a graph with new inputs
    M, K = 64, 2048
    X, res, w = _values((M, K), 51, torch.bfloat16), _values((M, K), 52, torch.bfloat16), torch.ones(K, device=DEV)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        x2 = X * 2
        Y, out = L.add_rms_norm(x2, w, 1e-5, residual=res)
        Z = L.gated_activation(out, x2)
    torch.cuda.current_stream().wait_stream(s)
    Y1, out1 = L.add_rms_norm(X * 2, w, 1e-5, residual=res)
    assert torch.equal(Y, Y1) and torch.equal(out, out1) and torch.equal(Z, L.gated_activation(out1, X * 2))
    static, r = X.clone(), res.clone()
    Yg, h = torch.empty_like(Y), torch.empty_like(res)
    Zg = torch.empty_like(Z)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        L.add_rms_norm(static, w, 1e-5, residual=r, residual_out=h, Y=Yg)
        L.gated_activation(h, static, Y=Zg)
    for k in (3, 5):
        static.copy_(X * k)
        graph.replay()
        Y1, out1 = L.add_rms_norm(X * k, w, 1e-5, residual=res)
        assert torch.equal(Yg, Y1) and torch.equal(h, out1) and torch.equal(Zg, L.gated_activation(out1, X * k))


def test_the_public_ways_to_device_and_stream_say_the_same(monkeypatch):
    s = torch.cuda.Stream()
    for stream in (torch.cuda.current_stream(), s):
        with torch.cuda.stream(stream):
            assert binding._public_raw_stream(0) == binding._raw_stream(0) == stream.cuda_stream
    X, w = _values((3, 256), 81, torch.float32), torch.ones(256, device=DEV)
    Y, _ = L.add_rms_norm(X, w, 1e-5)
    monkeypatch.setattr(binding, "_raw_stream", binding._public_raw_stream)
    monkeypatch.setattr(binding, "_current_device", torch.cuda.current_device)
    assert torch.equal(L.add_rms_norm(X, w, 1e-5)[0], Y)


# ---- batches of prompt size: more rows than there are CTAs, so that a CTA works on one row with the next one on its way ----

@pytest.mark.parametrize("y", ["f32", "bf16", "mxint8"])
@pytest.mark.parametrize("r", ["f32", "bf16"])
@pytest.mark.parametrize("x", ["f32", "bf16"])
@pytest.mark.parametrize("M,K", [(5000, 48), (2500, 1040), (700, 4112), (601, 8208), (400, 16400)])
def test_add_rms_norm_of_a_prompt(M, K, x, r, y):
    X, res = _values((M, K), 91, TYPES[x], 3), _values((M, K), 92, TYPES[r], 3)
    w = 1.0 + 0.2 * _values((K,), 93, torch.float32, 0)
    out_dtype = L.MXINT8 if y == "mxint8" else TYPES[y]
    h = (X.float() + res.float()).to(TYPES[r])
    Y, out = L.add_rms_norm(X, w, 1e-5, residual=res, out_dtype=out_dtype)
    assert torch.equal(out, h)
    _check(Y, _norm64(h, w, 1e-5), 3 * U * (1 + 4 * U), M, K, y, _cfg())
    # the sum in the residual's place, or in X's: a row is written while the next one is on its way
    own = res.clone()
    Z, out = L.add_rms_norm(X, w, 1e-5, residual=own, residual_out=own, out_dtype=out_dtype)
    assert out is own and torch.equal(own, h) and torch.equal(Z, Y)
    if x == r:
        own = X.clone()
        Z, out = L.add_rms_norm(own, w, 1e-5, residual=res, residual_out=own, out_dtype=out_dtype)
        assert out is own and torch.equal(own, h) and torch.equal(Z, Y)
    # no residual, h not kept
    Z, out = L.add_rms_norm(h, w, 1e-5, out_dtype=out_dtype)
    assert out is None and torch.equal(Z, Y)


@pytest.mark.parametrize("y", ["f32", "bf16", "mxint8"])
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("x", ["f32", "bf16"])
@pytest.mark.parametrize("M,N,joined", [(2500, 272, True), (1500, 2064, False), (1301, 2064, True), (601, 11008, False), (250, 13824, True)])
def test_gated_activation_of_a_prompt(M, N, joined, x, act, y):
    if joined:
        both = _values((M, 2 * N), 94, TYPES[x], 3)
        gate, up = both[:, :N], both[:, N:]
    else:
        gate, up = _values((M, N), 94, TYPES[x], 3), _values((M, N), 95, TYPES[x], 3)
    cfg = _cfg(6 if M == 1301 else 8)
    Y = L.gated_activation(gate, up, act=act, out_dtype=L.MXINT8 if y == "mxint8" else TYPES[y], cfg=cfg)
    g = gate.double()
    z = g if act == "silu" else 2.0 * math.sqrt(2.0 / math.pi) * (g + 0.044715 * g ** 3)
    want = g / (1.0 + torch.exp(-z)) * up.double()
    zs = 0.0 if act == "silu" else z.abs().cpu().numpy()
    _check(Y, want.cpu().numpy(), (10 + 7 * zs) * U * (1 + 1e-5), M, N, y, cfg, tiny=2.0 ** -102)


def test_values_of_a_prompt():
    M, K = 2300, 11008                           # more blocks than the grid has threads
    g = torch.Generator(device=DEV).manual_seed(96)
    m = torch.randint(-127, 128, (M, K), generator=g, device=DEV, dtype=torch.int8)
    e = torch.randint(127 - 56, 127 + 56, (M, K // 16), generator=g, device=DEV, dtype=torch.uint8)
    want = m.double() * torch.exp2(e.double() - 127 - 6).repeat_interleave(16, 1)
    for dt in (torch.float32, torch.bfloat16):
        got = L.dequantize_activations(L.to_mxint8(m, e), M, K, out_dtype=dt)
        assert torch.equal(got.double(), want)
