"""Adapters of many requests beside a shared projection, against 64-bit arithmetic.

Bound of a row's result: with S = scale (|X| |A|) |B| the errors are relative to S.  fp32 X and T are cut to 16 bits for bf16 Y
(2^-16 each) and to 24 for fp32 Y (2^-23 each; the parts of X hold all of it).  An MMA may cut its running sum at 2^-22 of its
magnitude; a sum of T passes through at most K / 16 MMAs a part and 16 partial sums, one of Y through rank / 16 MMAs a part.  The
scale and the last addition are rounded (2^-24 each, of S and of the result), and a bf16 result (2^-8).
"""
import os
import subprocess
import sys
import textwrap

import numpy as np
import pytest
import torch

import paper_2402_02446_b200 as L

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BAD_PACKED, TIMEOUT, BOUNDS = 6, 9, 10
FAM_DECODE = 7


def _randn(shape, seed, dtype=torch.float32):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randn(shape, generator=g, device=DEV).to(dtype)


class Case:
    def __init__(self, M, K, N, ranks, slots, x="bf16", y0="f32", y="f32", seed=0, max_rank=None, load=torch.bfloat16):
        self.M, self.K, self.N, self.kinds = M, K, N, (x, y0, y)
        self.A = [_randn((K, r), seed + 10 + 2 * j, torch.bfloat16) if r else None for j, r in enumerate(ranks)]
        self.B = [_randn((r, N), seed + 11 + 2 * j, torch.bfloat16) if r else None for j, r in enumerate(ranks)]
        self.scale = [0.25 + 0.5 * j for j in range(len(ranks))]
        self.pool = L.new_adapter_pool(K, N, max_rank or max(max(ranks), 1), len(ranks))
        for j, r in enumerate(ranks):
            if r:
                L.load_adapter(self.pool, j, self.A[j].to(load), self.B[j].to(load), self.scale[j])
        self.slots = torch.tensor(slots, dtype=torch.int32, device=DEV)
        X = _randn((M, K), seed + 1) * torch.exp2(torch.randint(-3, 4, (M, K // 16), generator=torch.Generator().manual_seed(seed)).float().to(DEV).repeat_interleave(16, 1))
        if x == "mxint8":
            self.X = L.to_mxint8(*L.quantize_activations(X))
            self.X64 = L.dequantize_activations(self.X, M, K).double()
        else:
            self.X = X.to(TYPES[x])
            self.X64 = self.X.double()
        self.Y0 = (_randn((M, N), seed + 2) * K ** 0.5).to(TYPES[y0])

    def run(self, Y=None):
        self.plan = L.adapter_plan(self.slots, self.pool)
        Y = L.apply_adapters(self.X, self.pool, self.plan, self.Y0, Y=Y, out_dtype=TYPES[self.kinds[2]])
        return Y

    def check(self, Y, slots=None):
        x, _, y = self.kinds
        want, S = self.Y0.double(), torch.zeros_like(self.Y0, dtype=torch.float64)
        parts = 3 if y == "f32" else 2
        rank = 0
        for j, (A, B) in enumerate(zip(self.A, self.B)):
            at = ((self.slots if slots is None else slots) == j).nonzero()[:, 0]
            if A is not None and len(at):
                rank = max(rank, A.shape[1])
                want[at] += self.scale[j] * ((self.X64[at] @ A.double()) @ B.double())
                S[at] += self.scale[j] * ((self.X64[at].abs() @ A.double().abs()) @ B.double().abs())
        cut = 2.0 ** -23 if y == "f32" else 2.0 ** -16
        mmas = (self.K // 16 + 1) * (parts if x == "f32" else 1) + 16 + (rank // 16 + 1) * parts
        bound = S * (2 * cut + mmas * 2.0 ** -22 + 2.0 ** -24) * 1.001 + want.abs() * (2.0 ** -24 + (2.0 ** -8 * 1.01 if y == "bf16" else 0.0))
        assert Y.dtype == TYPES[y]
        off = (Y.double() - want).abs()
        assert bool((off <= bound).all()), float((off / bound).nan_to_num(nan=9e9).max())
        bare = S.sum(1) == 0                     # rows without an adapter come through as they are
        if bare.any():
            assert torch.equal(Y[bare], self.Y0[bare].to(Y.dtype))


SHAPES = [
    # M, K, N, ranks, slots of the rows
    (1, 256, 256, [8], [0]),
    (1, 4096, 4096, [16], [0]),
    (2, 272, 264, [1, 5], [1, 0]),
    (16, 1040, 1048, [16, 4, 64, 20], [0, 1, 2, 3, -1, 3, 2, 1, 0, 0, 0, 3, 3, -1, -1, 2]),
    (17, 512, 520, [64], [0] * 17),
    (40, 2064, 2080, [100, 128, 8], [j % 4 - 1 for j in range(40)]),
    (3, 528, 536, [256, 200], [0, 1, 0]),
    (33, 16, 8, [8, 3], [j % 3 - 1 for j in range(33)]),
    (201, 4112, 1096, [20] * 8, [j // 30 - 1 for j in range(201)]),
]


@pytest.mark.parametrize("x,y0,y", [("bf16", "bf16", "bf16"), ("f32", "f32", "f32"), ("mxint8", "f32", "f32"), ("bf16", "f32", "f32"),
                                    ("f32", "f32", "bf16"), ("mxint8", "bf16", "bf16"), ("bf16", "bf16", "f32")])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"M{s[0]}_K{s[1]}_N{s[2]}_r{max(s[3])}")
def test_adapters(shape, x, y0, y):
    c = Case(*shape, x=x, y0=y0, y=y)
    Y = c.run()
    assert L.poll_status(c.plan.buf) == 0
    c.check(Y)


@pytest.mark.parametrize("x,y", [("bf16", "bf16"), ("f32", "f32"), ("mxint8", "bf16"), ("bf16", "f32"), ("f32", "bf16"), ("mxint8", "f32")])
@pytest.mark.parametrize("M,ranks", [(513, [16, 8]), (700, [64, 33, 5]), (1300, [128]), (530, [256, 8]), (1025, [16, 3]), (1100, [256, 20]), (2500, [32, 8, 17]),
                                     (1040, [256, 256])])
def test_adapters_many_rows(M, ranks, x, y):
    # runs of uneven length, scattered rows and rows without adapter; up to 1024 rows of products as small as these are "few"
    g = torch.Generator().manual_seed(M)
    slots = torch.sort(torch.randint(-1, len(ranks), (M,), generator=g))[0]
    slots[::7] = torch.randint(-1, len(ranks), (len(slots[::7]),), generator=g)
    c = Case(M, 1040, 1064, ranks, slots.tolist(), x=x, y0=y, y=y)
    Y = c.run()
    assert L.poll_status(c.plan.buf) == 0
    c.check(Y)


def test_random_batches_of_many_slots():
    g = torch.Generator().manual_seed(3)
    for M, n in ((1, 64), (7, 1024), (64, 64), (129, 3), (512, 1000), (515, 600), (1024, 1024), (1500, 900), (4097, 1024)):
        slots = torch.randint(-1, n, (M,), generator=g).tolist()
        ranks = [(j * 7) % 17 for j in range(n)]              # empty slots among them
        c = Case(M, 64, 72, ranks, slots, max_rank=16)
        c.check(c.run())
        assert L.poll_status(c.plan.buf) == 0


def test_a_row_does_not_depend_on_its_neighbours():
    c = Case(48, 1040, 520, [16, 32], [j % 3 - 1 for j in range(48)])
    Y = c.run()
    perm = torch.randperm(48, generator=torch.Generator().manual_seed(4)).to(DEV)
    c.slots, c.X, c.X64, c.Y0 = c.slots[perm].contiguous(), c.X[perm].contiguous(), c.X64[perm], c.Y0[perm].contiguous()
    assert torch.equal(c.run(), Y[perm])
    # a row of NaN and infinities stays alone
    c.X[5] = float("nan")
    c.X[6, 3] = float("inf")
    Z = c.run()
    keep = torch.ones(48, dtype=torch.bool, device=DEV)
    keep[5] = keep[6] = False
    assert torch.equal(Z[keep], Y[perm][keep])
    if c.slots[5] >= 0:
        assert torch.isnan(Z[5]).all()


@pytest.mark.parametrize("x", ["f32", "bf16"])
def test_infinities_and_the_largest_values(x):
    # an infinite or largest-possible activation gives what the products give: no NaN from its parts or from the rank's padding
    c = Case(4, 64, 32, [5], [0, 0, 0, -1], x=x, y0="f32", y="f32")
    c.X[:] = 0
    c.X[0, 3] = float("inf")
    c.X[1, 3] = -float("inf")
    c.X[2, 3] = torch.finfo(c.X.dtype).max
    L.load_adapter(c.pool, 0, torch.full((64, 5), 2.0 ** -20, device=DEV), torch.ones((5, 32), device=DEV), 1.0)
    Y = c.run()
    assert (Y[0] == float("inf")).all() and (Y[1] == -float("inf")).all()
    want = c.Y0[2].double() + c.X[2, 3].double() * 2.0 ** -20 * 5
    assert torch.allclose(Y[2].double(), want, rtol=2.0 ** -20)
    assert torch.equal(Y[3], c.Y0[3])


def test_in_place_and_given_outputs():
    slots = [0, -1, 1, 1, 0, -1]
    for y in ("f32", "bf16"):
        c = Case(6, 512, 264, [16, 8], slots, y0=y, y=y)
        Y = c.run()
        Z = torch.full_like(Y, 3.0)
        assert c.run(Y=Z) is Z and torch.equal(Z, Y)
        inplace = c.Y0.clone()
        L.apply_adapters(c.X, c.pool, c.plan, inplace, Y=inplace)
        assert torch.equal(inplace, Y)
        c.check(Y)


@pytest.mark.parametrize("M", [3, 40, 1100])
def test_activations_of_another_format(M):
    # six bits, a window that saturates large blocks and drops small ones: the values are those that the layer would take
    cfg = L.default_config()
    cfg.a_bits, cfg.exp_min, cfg.exp_max = 6, -3, 1
    c = Case(M, 528, 264, [16, 40], [j % 3 - 1 for j in range(M)])
    X = _randn((M, 528), 31) * torch.exp2(torch.arange(33, device=DEV) % 9 - 6.0).repeat_interleave(16)
    Xq = L.to_mxint8(*L.quantize_activations(X, cfg=cfg))
    c.X64, c.kinds = L.dequantize_activations(Xq, M, 528, cfg=cfg).double(), ("mxint8", "f32", "f32")
    plan = L.adapter_plan(c.slots, c.pool)
    c.check(L.apply_adapters(Xq, c.pool, plan, c.Y0, cfg=cfg))


@pytest.mark.parametrize("x,y", [("f32", "f32"), ("bf16", "bf16"), ("mxint8", "f32")])
def test_few_rows_of_tensors_aligned_to_16_bytes_only(x, y):
    def shifted(t):
        n = 16 // t.element_size()
        return torch.empty(t.numel() + 2 * n, dtype=t.dtype, device=DEV)[n:n + t.numel()].view(t.shape).copy_(t)
    c = Case(21, 528, 264, [16, 40], [j % 3 - 1 for j in range(21)], x=x, y0=y, y=y)
    Y = c.run()
    X, Y0, Z = shifted(c.X), shifted(c.Y0), shifted(c.Y0)
    assert X.data_ptr() % 32 == 16 and torch.equal(L.apply_adapters(X, c.pool, c.plan, Y0, Y=Z), Y)


def test_fp32_factors_are_rounded_to_bf16_and_slots_are_replaced():
    c = Case(5, 256, 256, [16, 8], [0, 1, 0, 1, 0], load=torch.float32)
    c.check(c.run())
    # a slot emptied, and loaded again with another rank; wider than bf16 holds, so rounded (nearest even)
    L.unload_adapter(c.pool, 0)
    Y = c.run()
    assert torch.equal(Y[0::2], c.Y0[0::2]) and L.poll_status(c.plan.buf) == 0
    A, B = _randn((256, 5), 91), _randn((5, 256), 92)
    c.A[0], c.B[0], c.scale[0] = A.bfloat16(), B.bfloat16(), -2.0
    L.load_adapter(c.pool, 0, A, B, -2.0)
    Y = c.run()
    c.scale[0] = 2.0
    c.A[0] = -c.A[0]
    c.check(Y)


def test_bad_slots_plans_and_pools_are_reported_and_touch_nothing():
    c = Case(20, 256, 264, [8, 16, 8, 8], [0, 1, 4, -2, 2 ** 31 - 1, -2 ** 31] + [3] * 14)
    Y = c.run()
    assert L.poll_status(c.plan.buf) == BOUNDS
    assert torch.equal(Y[2:6], c.Y0[2:6])
    fixed = c.slots.clone()
    fixed[2:6] = -1
    c.check(Y, fixed)
    # a buffer that no plan was made in, and one of another batch: nothing is written
    for buf in (torch.zeros_like(c.plan.buf), torch.full_like(c.plan.buf, 255)):
        buf[:16] = 0
        Z = torch.full_like(Y, 5.0)
        L.apply_adapters(c.X, c.pool, L.AdapterPlan(buf, 20, 4), c.Y0, Y=Z)
        assert L.poll_status(buf) == BAD_PACKED and (Z == 5.0).all()
    small = L.adapter_plan(c.slots[:19].contiguous(), c.pool)
    big = torch.zeros_like(c.plan.buf)
    big[:small.buf.numel()] = small.buf[:big.numel()]
    Z = torch.full_like(Y, 5.0)
    L.apply_adapters(c.X, c.pool, L.AdapterPlan(big, 20, 4), c.Y0, Y=Z)
    assert L.poll_status(big) in (BAD_PACKED, BOUNDS) and (Z == 5.0).all()
    # a pool that was not emptied first: its slots are unknown, rows take no adapter
    p = L.AdapterPool(256, 264, 16, 4, DEV)
    p.buf.fill_(171)
    plan = L.adapter_plan(torch.zeros(20, dtype=torch.int32, device=DEV), p)
    Z = L.apply_adapters(c.X, p, plan, c.Y0)
    assert L.poll_status(plan.buf) == BAD_PACKED and torch.equal(Z, c.Y0)


@pytest.mark.parametrize("M", [2, 512, 1024, 2000])
def test_a_shorter_batchs_plan_is_refused_unread(M):
    # the plan's buffer holds one row's lists and no more; the call would need some hundred times as much
    c = Case(M, 256, 264, [8, 16, 8, 8], [j % 5 - 1 for j in range(M)])
    small = L.adapter_plan(c.slots[:1], c.pool)
    Z = torch.full_like(c.Y0, 5.0)
    L.apply_adapters(c.X, c.pool, L.AdapterPlan(small.buf, M, 4), c.Y0, Y=Z)
    assert L.poll_status(small.buf) == BAD_PACKED and (Z == 5.0).all()
    c.check(c.run())


def test_streams_graphs_and_two_batches_at_once():
    c = Case(24, 1040, 520, [16, 64, 8], [j % 4 - 1 for j in range(24)])
    Y = c.run()
    # a graph that sorts the rows and applies the adapters; its replays follow the slots and the activations
    slots, X, Z = c.slots.clone(), c.X.clone(), torch.empty_like(Y)
    plan = L.adapter_plan(slots, c.pool)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        L.adapter_plan(slots, c.pool, plan=plan)
        L.apply_adapters(X, c.pool, plan, c.Y0, Y=Z)
    graph.replay()
    assert torch.equal(Z, Y)
    slots.copy_(c.slots.flip(0))
    X.copy_(c.X * 2)
    graph.replay()
    c.slots, c.X, c.X64 = slots, X, X.double()
    c.check(Z)
    # two batches on two streams share the pool, each with a plan of its own
    d = Case(300, 1040, 520, [16, 64, 8], [j // 80 - 1 for j in range(300)], seed=500)
    d.pool, d.A, d.B, d.scale = c.pool, c.A, c.B, c.scale
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    got = []
    for _ in range(10):
        with torch.cuda.stream(s1):
            got.append((c, c.run()))
        with torch.cuda.stream(s2):
            got.append((d, d.run()))
    torch.cuda.synchronize()
    for case, Yk in got:
        case.check(Yk)


def _many(seed=0, y="bf16", M=1500, ranks=(64, 16, 0, 40), K=1040, N=1064):
    """A batch that takes the tensor-core kernels: runs, scattered rows, rows without an adapter and rows of an empty slot."""
    g = torch.Generator().manual_seed(seed)
    slots = torch.sort(torch.randint(-1, len(ranks), (M,), generator=g))[0]
    slots[::9] = torch.randint(-1, len(ranks), (len(slots[::9]),), generator=g)
    c = Case(M, K, N, list(ranks), slots.tolist(), x=y, y0=y, y=y, seed=seed, max_rank=64)
    assert L.adapters_workspace_bytes(M, c.pool) > 0
    return c


@pytest.mark.parametrize("y", ["f32", "bf16"])
def test_many_rows_in_place_and_the_same_again(y):
    c = _many(1, y)
    Y = c.run()
    c.check(Y)
    inplace = c.Y0.clone()
    L.apply_adapters(c.X, c.pool, c.plan, inplace, Y=inplace)
    assert torch.equal(inplace, Y)
    # whichever CTA takes which columns, the results are the same
    ws = torch.full((L.adapters_workspace_bytes(c.M, c.pool),), 255, dtype=torch.uint8, device=DEV)
    for _ in range(5):
        assert torch.equal(L.apply_adapters(c.X, c.pool, c.plan, c.Y0, ws=ws), Y)
    # tensors that are aligned to 16 bytes only
    def shifted(t):
        n = 16 // t.element_size()
        return torch.empty(t.numel() + 2 * n, dtype=t.dtype, device=DEV)[n:n + t.numel()].view(t.shape).copy_(t)
    X, Y0, Z = shifted(c.X), shifted(c.Y0), shifted(c.Y0)
    assert X.data_ptr() % 32 == 16 and torch.equal(L.apply_adapters(X, c.pool, c.plan, Y0, Y=Z), Y)


@pytest.mark.parametrize("x,y0,y", [("f32", "f32", "f32"), ("bf16", "bf16", "bf16"), ("mxint8", "f32", "bf16"), ("bf16", "bf16", "f32")])
@pytest.mark.parametrize("M,K,N,ranks", [(1500, 272, 11016, [64, 0, 20]), (1500, 272, 11016, [128, 0, 20]), (1100, 48, 20488, [8, 256])])
def test_many_columns(M, K, N, ranks, x, y0, y):
    # many groups of columns to a CTA, the first two of them neighbours; an empty slot, rows without adapter
    c = Case(M, K, N, ranks, [(j // 37) % (len(ranks) + 1) - 1 for j in range(M)], x=x, y0=y0, y=y)
    Y = c.run()
    assert L.poll_status(c.plan.buf) == 0
    c.check(Y)


@pytest.mark.parametrize("x", ["f32", "bf16", "mxint8"])
@pytest.mark.parametrize("M,K,N,rank", [(4500, 10256, 264, 24), (12700, 2064, 136, 16), (2100, 16400, 72, 256)])
def test_long_projections(M, K, N, rank, x):
    # stretches of more slabs than an accumulator takes at a time, and stretches that end in the middle of a tile
    c = Case(M, K, N, [rank, 8], [(j // 300) % 3 - 1 for j in range(M)], x=x, y0="f32", y="f32")
    Y = c.run()
    assert L.poll_status(c.plan.buf) == 0
    c.check(Y)


def test_many_rows_without_any_adapter():
    c = _many(2)
    c.slots.fill_(-1)
    assert torch.equal(c.run(), c.Y0)
    inplace = c.Y0.clone()
    L.apply_adapters(c.X, c.pool, c.plan, inplace, Y=inplace)
    assert torch.equal(inplace, c.Y0)
    for j in range(4):
        L.unload_adapter(c.pool, j)
    c.slots[:] = torch.arange(c.M, device=DEV) % 4
    assert torch.equal(c.run(), c.Y0) and L.poll_status(c.plan.buf) == 0
    c.pool.buf[:32] = 255                                      # a slot that nobody wrote
    assert torch.equal(c.run(), c.Y0) and L.poll_status(c.plan.buf) == BAD_PACKED


def test_many_rows_next_to_a_row_of_nan():
    c = _many(3)
    Y = c.run()
    c.X[700] = float("nan")
    c.X[701, 5] = float("inf")
    Z = c.run()
    keep = torch.ones(c.M, dtype=torch.bool, device=DEV)
    keep[700] = keep[701] = False
    assert torch.equal(Z[keep], Y[keep])


def test_many_rows_streams_and_graphs():
    c, d = _many(4), _many(500, "f32", M=1100)
    Yc, Yd = c.run(), d.run()
    slots, X, Z = c.slots.clone(), c.X.clone(), torch.empty_like(Yc)
    plan = L.adapter_plan(slots, c.pool)
    ws = torch.empty(L.adapters_workspace_bytes(c.M, c.pool), dtype=torch.uint8, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        L.adapter_plan(slots, c.pool, plan=plan)
        L.apply_adapters(X, c.pool, plan, c.Y0, Y=Z, ws=ws)
    graph.replay()
    assert torch.equal(Z, Yc)
    slots.copy_(c.slots.flip(0))
    X.copy_(c.X * 2)
    graph.replay()
    graph.replay()
    old = c.slots, c.X, c.X64
    c.slots, c.X, c.X64 = slots, X, X.double()
    c.check(Z)
    c.slots, c.X, c.X64 = old
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    got = []
    for _ in range(6):
        with torch.cuda.stream(s1):
            got.append((Yc, c.run()))
        with torch.cuda.stream(s2):
            got.append((Yd, d.run()))
    torch.cuda.synchronize()
    for want, have in got:
        assert torch.equal(have, want)


def test_a_given_stream_owns_what_the_calls_make():
    # workspace and outputs come from the stream that is given: what the current one makes meanwhile lies elsewhere
    c = _many(8, "f32")
    Y = c.run()
    s = torch.cuda.Stream()
    for _ in range(3):
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            torch.cuda._sleep(2_000_000)
        pool = L.new_adapter_pool(1040, 1064, 64, 4, stream=s)
        plan = L.adapter_plan(c.slots, c.pool, stream=s)
        Z = L.apply_adapters(c.X, c.pool, plan, c.Y0, stream=s)
        W = L.apply_adapters(c.X, pool, plan, c.Y0, stream=s)
        waste = [torch.full((n,), 255, dtype=torch.uint8, device=DEV) for n in (L.adapters_workspace_bytes(c.M, c.pool), plan.buf.numel(), Y.numel() * 4)]
        s.synchronize()
        assert torch.equal(Z, Y) and torch.equal(W, c.Y0) and L.poll_status(plan.buf) == 0
        del waste


def test_many_rows_behind_the_kernel_that_makes_their_input():
    # the kernels overlap their neighbours on the stream: inputs made, used, and made anew without a pause
    c = _many(6, "f32")
    want = [L.apply_adapters(c.X * k, c.pool, L.adapter_plan(c.slots, c.pool), c.Y0 * k) for k in (1, 2, 4)]
    torch.cuda.synchronize()
    plan, X, Y0 = L.adapter_plan(c.slots, c.pool), torch.empty_like(c.X), torch.empty_like(c.Y0)
    w = torch.ones(1040, device=DEV)
    for _ in range(4):
        got = []
        for k in (1, 2, 4):
            L.adapter_plan(c.slots, c.pool, plan=plan)
            torch.mul(c.X, k, out=X)
            torch.mul(c.Y0, k, out=Y0)
            got.append(L.apply_adapters(X, c.pool, plan, Y0))
            L.add_rms_norm(X, w, 1e-5)
        for a, b in zip(got, want):
            assert torch.equal(a, b)


def test_a_wait_that_runs_out_is_reported_and_the_next_call_is_fine():
    c = _many(7)
    Y = c.run()
    L.set_wait_limit_cycles(2_000_000)                          # about a millisecond
    L.inject_stall(FAM_DECODE)
    try:
        c.run()
        torch.cuda.synchronize()
    finally:
        L.inject_stall(-1)
        L.set_wait_limit_cycles(4_000_000_000)
    assert L.poll_status(c.plan.buf) == TIMEOUT
    for _ in range(2):
        assert torch.equal(c.run(), Y) and L.poll_status(c.plan.buf) == 0


@pytest.mark.parametrize("y", ["f32", "bf16"])
def test_waits_that_run_out_anywhere_leave_nothing_under_way(y):
    # bounds around the time that ordinary waits take: now one role gives up, now another, with copies and products on their way;
    # the calls that follow own the same shared and tensor memory
    c = _many(11, y, M=3000, N=2056)
    Y = c.run()
    c.check(Y)
    for limit in (1000, 1500, 2500, 4000, 6000, 10000, 20000) * 3:
        L.set_wait_limit_cycles(limit)
        try:
            Z = c.run()
            torch.cuda.synchronize()
        finally:
            L.set_wait_limit_cycles(4_000_000_000)
        status = L.poll_status(c.plan.buf)
        assert status in (0, TIMEOUT) and (status != 0 or torch.equal(Z, Y))
        assert torch.equal(c.run(), Y) and L.poll_status(c.plan.buf) == 0


def test_the_checked_build_keeps_to_the_extent_of_y():
    code = textwrap.dedent("""
        import sys, torch
        sys.path.insert(0, "tests")
        import test_gpu_adapters as t
        import paper_2402_02446_b200 as L
        from paper_2402_02446_b200 import binding
        assert binding.DEBUG_BOUNDS
        for y in ("f32", "bf16"):
            for c in (t.Case(20, 256, 264, [8, 16], [0, 1] * 10, x="bf16", y0=y, y=y), t._many(9, y)):
                Y = c.run()
                assert L.poll_status(c.plan.buf) == 0
                c.check(Y)
                Z = torch.full_like(Y, 7.0)
                L.debug_bounds_shrink(400)
                try:
                    c.run(Y=Z)
                    torch.cuda.synchronize()
                finally:
                    L.debug_bounds_shrink(0)
                assert L.poll_status(c.plan.buf) == t.BOUNDS
                n = 400 // Y.element_size()
                assert (Z.flatten()[-n:] == 7.0).all() and torch.equal(Z.flatten()[:-n - 16], Y.flatten()[:-n - 16])
        print("fine")
    """)
    r = subprocess.run([sys.executable, "-c", code], cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                       env=dict(os.environ, LQER_DEBUG_BOUNDS="1"), capture_output=True, text=True, timeout=600)
    assert r.returncode == 0 and "fine" in r.stdout, r.stdout[-1500:] + r.stderr[-2500:]


def test_a_block_of_layers_with_adapters():
    """Norm, two adapted layers, the gate, an adapted layer, the next norm: as a serving program runs them, against 64 bits."""
    import lqer_inputs as gen
    from oracle import lqer as olqer
    from oracle import mxint
    M, K, F = 21, 256, 528
    g = np.random.default_rng(8)
    layers = {}
    for name, k_in, n_out in (("gate", K, F), ("up", K, F), ("down", F, K)):
        spec = gen.LayerSpec(name, M=M, K=k_in, N=n_out, k=16, calib_rows=32, outlier_frac=0.0, outlier_scale=1.0, seed=len(name))
        W = gen.make_weight(spec)
        A, B = gen.make_random_factors(spec)
        P = L.prepare_weights(*(torch.from_numpy(np.ascontiguousarray(v)).to(DEV) for v in (W, A, B)))
        pool = L.new_adapter_pool(k_in, n_out, 8, 3)
        lora = []
        for j in range(3):
            a = _randn((k_in, 8), 100 + j, torch.bfloat16) * k_in ** -0.5
            b = _randn((8, n_out), 200 + j, torch.bfloat16) * 0.1
            L.load_adapter(pool, j, a, b, 0.5)
            lora.append((a.double().cpu().numpy(), b.double().cpu().numpy()))
        layers[name] = (olqer.prepare_weights(W, A, B), P, pool, lora)
    slots = g.integers(-1, 3, M).astype(np.int32)
    plan = L.adapter_plan(torch.from_numpy(slots).to(DEV), layers["gate"][2])
    ws = max((L.new_workspace(M, P) for _, P, _, _ in layers.values()), key=lambda t: t.numel())
    x, res, w = _randn((M, K), 1), _randn((M, K), 2), 1 + 0.1 * _randn((K,), 3)
    xq, h = L.add_rms_norm(x, w, 1e-5, residual=res)
    outs = {}
    for name in ("gate", "up"):
        y = L.linear_ex(xq, layers[name][1], ws, M=M)
        outs[name] = L.apply_adapters(xq, layers[name][2], plan, y, Y=y)
    aq = L.gated_activation(outs["gate"], outs["up"])
    y = L.linear_ex(aq, layers["down"][1], ws, M=M)
    y = L.apply_adapters(aq, layers["down"][2], plan, y, Y=y)
    last, h2 = L.add_rms_norm(y, w, 1e-5, residual=h, out_dtype=torch.float32)
    assert L.poll_status(ws) == 0 and L.poll_status(plan.buf) == 0

    # each step against 64 bits from the step's own inputs (a quantiser in between would turn a last bit into a step)
    def adapted(name, q, got):
        prep, _, _, lora = layers[name]
        v = L.dequantize_activations(q, M, prep.K).double().cpu().numpy()
        ref = olqer.forward(v.astype(np.float32), prep)
        want, tol = ref.Y.copy(), ref.tol.copy()
        for m in range(M):
            if slots[m] >= 0:
                a, b = lora[slots[m]]
                want[m] += 0.5 * (v[m] @ a) @ b
                tol[m] += 1e-4 * 0.5 * (np.abs(v[m]) @ np.abs(a)) @ np.abs(b)
        assert np.all(np.abs(got.double().cpu().numpy() - want) <= tol + 2.0 ** -23 * np.abs(want))
    adapted("gate", xq, outs["gate"])
    adapted("up", xq, outs["up"])
    adapted("down", aq, y)
    h64 = (x + res).double().cpu().numpy()
    m, e = mxint.quantize(h64 / np.sqrt((h64 ** 2).mean(1, keepdims=True) + 1e-5) * w.double().cpu().numpy(), 8, 1)
    assert np.array_equal(L.dequantize_activations(xq, M, K).double().cpu().numpy(), mxint.dequantize(m, e, 8, 1))
    a64, b64 = outs["gate"].double().cpu().numpy(), outs["up"].double().cpu().numpy()
    m, e = mxint.quantize(a64 / (1 + np.exp(-a64)) * b64, 8, 1)
    assert np.array_equal(L.dequantize_activations(aq, M, F).double().cpu().numpy(), mxint.dequantize(m, e, 8, 1))
    h64 = (y + h).double().cpu().numpy()
    want = h64 / np.sqrt((h64 ** 2).mean(1, keepdims=True) + 1e-5) * w.double().cpu().numpy()
    assert torch.equal(h2, y + h) and np.all(np.abs(last.double().cpu().numpy() - want) <= np.abs(want) * 2.0 ** -22)
    for _, P, _, _ in layers.values():
        P.release()
