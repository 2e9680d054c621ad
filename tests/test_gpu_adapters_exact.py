"""Adapters on whole numbers, where every sum is exact: a lost part of a number, a lost slab of K or a lost adapter shows in the last bit.

All sums stay below 2^21 in magnitude (checked on the absolute values), so fp32 sums and the tensor cores' (which may cut a running sum at 2^-22 of its
magnitude) hold them exactly, in any order.  Column n of B picks rank n % rank, except where B is given.
"""
import pytest
import torch

import paper_2402_02446_b200 as L

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _whole(shape, most, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randint(-most, most + 1, shape, generator=g, device=DEV).double()


def _picks(rank, N):
    B = torch.zeros((rank, N), dtype=torch.float64, device=DEV)
    n = torch.arange(N, device=DEV)
    B[n % rank, n] = 1.0
    return B


def _apply(X, As, Bs, slots, Y0, x, y):
    """The term of whole-number fp64 X, A, B through the library: Y as fp64, and the exact term."""
    M, K = X.shape
    pool = L.new_adapter_pool(K, Bs[0].shape[1], max(A.shape[1] for A in As), len(As))
    want = torch.zeros_like(Y0)
    for j, (A, B) in enumerate(zip(As, Bs)):
        assert (A.bfloat16().double() == A).all() and (B.bfloat16().double() == B).all()
        L.load_adapter(pool, j, A.bfloat16(), B.bfloat16(), 1.0)
        at = (slots == j).nonzero()[:, 0]
        S = (X[at].abs() @ A.abs()) @ B.abs()
        assert not len(at) or S.max() < 2.0 ** 21
        want[at] = (X[at] @ A) @ B
    if x == "mxint8":
        Xt = L.to_mxint8(*L.quantize_activations(X.float()))
        assert (L.dequantize_activations(Xt, M, K).double() == X).all()
    else:
        Xt = X.to(TYPES[x])
        assert (Xt.double() == X).all()
    plan = L.adapter_plan(slots.to(torch.int32), pool)
    Y = L.apply_adapters(Xt, pool, plan, Y0.float(), out_dtype=TYPES[y])
    assert L.poll_status(plan.buf) == 0
    return Y.double(), want


SHAPES = [(1, 64, 16), (2, 272, 5), (3, 272, 16), (24, 272, 100), (37, 64, 256), (600, 528, 16), (1100, 64, 16), (1100, 272, 100), (1100, 272, 256)]


def _batch(M, K, rank, x):
    X = _whole((M, K), 63, 1)
    if x == "mxint8":
        X[:, ::16] = 127.0                       # every block's step is one
    As = [_whole((K, rank), 15, 2), _whole((K, max(rank // 3, 1)), 15, 3)]
    slots = (torch.arange(M, device=DEV) // 5) % 3 - (1 if M > 5 else 0)
    return X, As, [_picks(A.shape[1], 264) for A in As], slots


@pytest.mark.parametrize("x", ["f32", "bf16", "mxint8"])
@pytest.mark.parametrize("M,K,rank", SHAPES)
def test_whole_numbers_are_exact_in_fp32(M, K, rank, x):
    X, As, Bs, slots = _batch(M, K, rank, x)
    Y0 = _whole((M, 264), 1000, 4)
    Y, want = _apply(X, As, Bs, slots, Y0, x, "f32")
    assert torch.equal(Y, Y0 + want)


def _shown(X, As, Bs, slots, x):
    """bf16 results beside an fp32 Y0 that cancels the term: what was rounded on the way, itself within half a step of bf16 (2^-8)."""
    want = torch.zeros((X.shape[0], Bs[0].shape[1]), dtype=torch.float64, device=DEV)
    for j, (A, B) in enumerate(zip(As, Bs)):
        at = (slots == j).nonzero()[:, 0]
        want[at] = (X[at] @ A) @ B
    Y, again = _apply(X, As, Bs, slots, -want, x, "bf16")
    assert torch.equal(again, want)
    return Y, want


@pytest.mark.parametrize("x", ["f32", "bf16", "mxint8"])
@pytest.mark.parametrize("M,_,rank", SHAPES)
def test_for_a_bf16_result_t_is_rounded_to_nearest(M, _, rank, x):
    # T, of 20 or 21 bits here, goes on as two bf16 parts, each rounded: 2^-9 of what the first can leave (2^-8)
    K = 144
    X = 64.0 + _whole((M, K), 31, 14).abs() * 2 + 1
    As = [64.0 + _whole((K, r), 31, 15).abs() * 2 for r in (rank, max(rank // 3, 1))]
    slots = (torch.arange(M, device=DEV) // 5) % 3 - (1 if M > 5 else 0)
    Y, T = _shown(X, As, [_picks(A.shape[1], 264) for A in As], slots, x)
    assert (Y.abs() <= T.abs() * 2.0 ** -17 * (1 + 2.0 ** -8)).all()


@pytest.mark.parametrize("M,rank", [(1, 16), (2, 16), (30, 16), (30, 100), (1100, 16), (1100, 100)])
def test_for_a_bf16_result_fp32_activations_are_rounded_to_nearest(M, rank):
    # A picks single activations of 20 bits: X as two parts, and T, which is that sum, as two parts again
    K = 272
    X = _whole((M, K), 2 ** 20, 5)
    A = torch.zeros((K, rank), dtype=torch.float64, device=DEV)
    A[torch.arange(rank, device=DEV) * 2 + 1, torch.arange(rank, device=DEV)] = 1.0
    Y, T = _shown(X, [A], [_picks(rank, 264)], torch.zeros(M, dtype=torch.int64, device=DEV), "f32")
    assert (Y.abs() <= T.abs() * 2 * 2.0 ** -17 * (1 + 2.0 ** -16) * (1 + 2.0 ** -8)).all()


@pytest.mark.parametrize("x", ["f32", "bf16", "mxint8"])
@pytest.mark.parametrize("M,K,N,rank", [(4500, 10256, 264, 24), (2100, 16400, 72, 256), (1100, 16400, 72, 128), (40, 16400, 72, 256), (600, 8208, 1048, 16)])
def test_long_sums_are_complete(M, K, N, rank, x):
    X = _whole((M, K), 1, 6)
    As = [_whole((K, rank), 1, 7), _whole((K, 8), 1, 8)]
    Bs = [_whole((rank, N), 1, 9), _whole((8, N), 1, 10)]
    slots = (torch.arange(M, device=DEV) // 300) % 3 - (1 if M > 900 else 0)
    Y0 = _whole((M, N), 1000, 11)
    Y, want = _apply(X, As, Bs, slots, Y0, x, "f32")
    assert torch.equal(Y, Y0 + want)


@pytest.mark.parametrize("M,K,rank", [(2, 1040, 16), (24, 1040, 24), (24, 16400, 256), (1100, 1040, 64), (2100, 16400, 24), (2100, 16400, 256)])
def test_the_lowest_bits_of_fp32_activations_survive_what_cancels(M, K, rank):
    # neighbours c + d and -c under one factor: only d is left, which lies in the lower parts of c + d
    d = _whole((M, K // 2), 3, 12)
    X = torch.stack([2.0 ** 17 + d, torch.full_like(d, -(2.0 ** 17))], 2).view(M, K)
    half = torch.zeros((K // 2, rank), dtype=torch.float64, device=DEV)
    at = torch.arange(K // 2, device=DEV)
    half[at, at % rank] = _whole((K // 2,), 1, 13)
    A, B = half.repeat_interleave(2, 0), _picks(rank, 264)
    slots = torch.zeros(M, dtype=torch.int64, device=DEV)
    pool = L.new_adapter_pool(K, 264, rank, 1)
    L.load_adapter(pool, 0, A.bfloat16(), B.bfloat16(), 1.0)
    plan = L.adapter_plan(slots.to(torch.int32), pool)
    Y = L.apply_adapters(X.float(), pool, plan, torch.zeros((M, 264), device=DEV))
    assert L.poll_status(plan.buf) == 0 and torch.equal(Y.double(), (d @ half) @ B)
