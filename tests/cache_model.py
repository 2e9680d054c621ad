"""A plain model of the paged cache for the tests: the tables in Python, the attention in 64 bits."""
from __future__ import annotations

import math

import torch

import paper_2402_02446_b200 as L


class Tables:
    """What cache_step has to make of lengths, tables, ring and added counts."""

    def __init__(self, R, max_pages, n_pages, page):
        self.R, self.max_pages, self.n_pages, self.page = R, max_pages, n_pages, page
        self.tables = [[-1] * max_pages for _ in range(R)]
        self.lengths = [0] * R
        self.free = list(range(n_pages))
        self.ring = [0, n_pages]

    def step(self, added, M, max_added):
        """(slots, positions, status, [(row0, n, length)]), the state stepping on."""
        P, status, cap = self.page, 0, self.max_pages * self.page
        SHORT, BOUNDS = 5, 10
        pages = lambda n: (n + P - 1) // P  # noqa: E731
        head, tail = self.ring
        plan, row = [], 0
        bad = []
        for ln, a in zip(self.lengths, added):
            nxt = max(0, ln + a)
            bad.append(ln < 0 or ln > cap or nxt > cap or a > max_added)
        give = sum(max(0, pages(ln) - pages(max(0, ln + a))) for ln, a, b in zip(self.lengths, added, bad) if not b)
        ring_ok = head >= 0 and tail >= head and tail - head + give <= self.n_pages
        ok = []
        for r, a in enumerate(added):
            ln, rows = self.lengths[r], max(a, 0)
            have, want = pages(ln), pages(max(0, ln + a))
            ok.append(not bad[r] and (row + rows <= M or rows == 0) and (ring_ok or have == want))
            if not ok[r]:
                status = status or BOUNDS
            plan.append([row, rows])
            row += rows
        if ring_ok:
            for r, a in enumerate(added):
                if not bad[r] and a < 0:
                    for c in range(pages(max(0, self.lengths[r] + a)), pages(self.lengths[r])):
                        self.free[tail % self.n_pages] = self.tables[r][c]
                        tail += 1
        avail, wanted, taken = (tail - head if ring_ok else 0), 0, 0
        for r, a in enumerate(added):
            have, want = pages(self.lengths[r]), pages(max(0, self.lengths[r] + a))
            if ok[r] and want > have:
                if wanted + want - have > avail:
                    ok[r] = False
                    status = SHORT if status == 0 else status
                else:
                    for c in range(have, want):
                        self.tables[r][c] = self.free[(head + wanted + c - have) % self.n_pages]
                    taken = wanted + want - have
                wanted += want - have
        slots, positions = [-1] * M, [-1] * M
        out = []
        for r, a in enumerate(added):
            row0, rows = plan[r]
            if ok[r]:
                for i in range(rows):
                    p = self.lengths[r] + i
                    slots[row0 + i], positions[row0 + i] = self.tables[r][p // P] * P + p % P, p
                self.lengths[r] = max(0, self.lengths[r] + a)
            out.append((row0, rows if ok[r] else 0, self.lengths[r]))
        self.ring = [head + taken, tail]
        return slots, positions, status, out


def cache_values(cache, cfg=None):
    """The keys and values of a cache [n_pages, kv_heads, page, head_dim] in 64 bits (on its device)."""
    shape = (cache.n_pages, cache.kv_heads, cache.page, cache.head_dim)
    if cache.dtype != L.MXINT8:
        return cache.keys.double(), cache.values.double()
    n = shape[0] * shape[1] * shape[2]
    return tuple(L.dequantize_activations(x, n, shape[3], cfg=cfg).double().view(shape) for x in (cache.keys, cache.values))


def attention64(Q, K, V, n, window, sinks, scale):
    """One request: Q [n, hq, D], K and V [hkv, len, D] in 64 bits.  (Y [n, hq, D], sum p |v| / sum p, the largest scale sum |q k|)."""
    hq, hkv, length = Q.shape[1], K.shape[0], K.shape[1]
    k, v = (x.repeat_interleave(hq // hkv, 0) for x in (K, V))
    s = torch.einsum("nhd,hld->hnl", Q, k) * scale
    most = (torch.einsum("nhd,hld->hnl", Q.abs(), k.abs()) * abs(scale)).amax()
    pos = torch.arange(length - n, length, device=Q.device)[:, None]
    j = torch.arange(length, device=Q.device)[None]
    seen = j <= pos
    if window:
        seen &= (j > pos - window) | (j < sinks)
    p = torch.softmax(s.masked_fill(~seen, -math.inf), -1)
    return torch.einsum("hnl,hld->nhd", p, v), torch.einsum("hnl,hld->nhd", p, v.abs()), float(most)


def tolerance(y, weighed, most, D, length):
    """Bound on |Y - y|.  The result is rounded to bf16 (2^-8 of it), and so are the weights (2^-8 of each; their sum is not).  The scores: D products
    summed in fp32, whose additions may cut off instead of rounding (2^-23 of the sums so far each), and three roundings more, an error of a score
    is one of its weight; exp2 is good to 2^-22, or, where a polynomial of third degree takes its
    place (prompts), to 7.5e-5: the largest |q(f) / 2^f - 1| over [-1/2, 1/2], with a few roundings of 2^-24.  Weights and sums over the tokens: 2^-23 for each addition, the joining of parts among them, as
    many again.  Errors of the weights count twice, in the sum of values and in the sum of weights."""
    weight = (D + 3) * 2.0 ** -23 * most + 7.6e-5
    return 2.0 ** -8 * y.abs() * 1.01 + (2.0 ** -8 + 2 * weight + 2 * length * 2.0 ** -23) * weighed * 1.01 + 2.0 ** -126


class Batch:
    """A cache and its tables, filled through the library in two steps: what the requests hold, and their new tokens, with anything where no token is."""

    def __init__(self, requests, hq, hkv, D, page, dtype=torch.bfloat16, pad=0, spare=3, x_dtype=torch.bfloat16, cfg=None, seed=0, max_added=None, scale=1.5,
                 dev="cuda:0", shuffle=True):
        self.requests, self.hq, self.hkv, self.D, self.cfg, self.dev = requests, hq, hkv, D, cfg, dev
        R = len(requests)
        pages = [(a + b + page - 1) // page for a, b in requests]
        n_pages, max_pages = sum(pages) + spare, max(max(pages), 1) + 1
        g = torch.Generator(device=dev).manual_seed(seed)
        rand = lambda *s: torch.randn(s, generator=g, device=dev)  # noqa: E731
        self.pages = L.new_page_table(R, max_pages, n_pages, page, device=dev)
        order = torch.arange(n_pages, device=dev, dtype=torch.int32)
        self.pages.free.copy_(order[torch.randperm(n_pages, generator=g, device=dev)] if shuffle else order.flip(0))
        self.cache = L.new_kv_cache(n_pages, page, hkv, D, dtype=dtype, device=dev)
        for t in (self.cache.keys, self.cache.values):
            t.fill_(float("nan")) if t.dtype == torch.bfloat16 else t.fill_(0xFF)
        before, new = [a for a, _ in requests], [b for _, b in requests]
        if sum(before):
            fill = L.cache_step(self.pages, torch.tensor(before, dtype=torch.int32, device=dev), sum(before))
            M = sum(before)
            L.append_kv(rand(M, hkv, D).to(x_dtype), rand(M, hkv, D).to(x_dtype), self.cache, fill.slots, cfg=cfg)
            assert L.poll_status(fill.buf) == 0
        self.M = max(1, sum(new) + pad)
        self.step = L.cache_step(self.pages, torch.tensor(new, dtype=torch.int32, device=dev), self.M, max_added=max_added or max(1, max(new)))
        both = rand(self.M, (hq + 2 * hkv) * D).to(x_dtype)
        L.append_kv(both[:, hq * D:(hq + hkv) * D], both[:, (hq + hkv) * D:], self.cache, self.step.slots, cfg=cfg)
        assert L.poll_status(self.step.buf) == 0
        self.Q = (both[:, :hq * D] * scale).to(torch.bfloat16).view(self.M, hq, D)

    def check(self, Y, window=0, sinks=0, scale=None, left=None, log=None, values=None):
        """Y against 64 bits, row by row; rows behind the last token hold `left` still.  values: gives pages' keys and values, where not all are wanted."""
        scale = self.D ** -0.5 if scale is None else scale
        if values is None:
            whole = cache_values(self.cache, self.cfg)
            values = lambda ids: tuple(x[ids] for x in whole)  # noqa: E731
        page, row, worst = self.pages.page, 0, 0.0
        for r, (before, n) in enumerate(self.requests):
            if n == 0:
                continue
            length = before + n
            ids = self.pages.tables[r, :(length + page - 1) // page].long()
            K, V = (x.transpose(0, 1).flatten(1, 2)[:, :length] for x in values(ids))
            y, weighed, most = attention64(self.Q[row:row + n].double(), K, V, n, window, sinks, scale)
            off = (Y[row:row + n].double() - y).abs() / tolerance(y, weighed, most, self.D, length)
            assert bool(torch.isfinite(Y[row:row + n]).all()), f"request {r}"
            worst = max(worst, float(off.max()))
            assert worst <= 1.0, (r, worst)
            row += n
        if left is not None:
            assert torch.equal(Y[row:], left[row:])
        if log is not None:
            log("attention", worst)
        return worst
