"""Operators over the keys and values of past tokens, as cases that can be timed and compared.

A case is one pass through one operator:

* ``step``    the tables of a paged cache brought from one step of a batch to the next (``cache_step``): pages given and taken
              back, and the slot and position of every new token;
* ``append``  the new tokens' keys and values into their slots (``append_kv``);
* ``decode``  attention of one or a few new tokens of each request over the cache (``paged_attention``);
* ``prompt``  attention of prompts, whole or in chunks behind what is cached, with or without a sliding window and first tokens
              that stay visible (``paged_attention``).

Hidden sizes are those of bench.py and of the test configurations with heads of 128 (4096: 32 heads, 5120: 40) and smaller ones, 1 to 8192
tokens a step, lengths that end inside a page or a tile.  An MXINT8 cache is handed back as the values that it stands for.

Each operator has a plain form in torch (``own`` False) next to the call of the library (``own`` True).
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
BLOCK = 16
EXP_MIN, EXP_MAX = -56, 55
BITS = 8
_FLOAT = {"f32": torch.float32, "bf16": torch.bfloat16}
_BYTES = {"f32": 4.0, "bf16": 2.0, "mxint8": 17.0 / 16.0}


def _step(R, longest, new, page, idle=0.0, done=0.0, drop=0):
    """R requests of up to `longest` tokens.  new: the tokens that each of them brings (of a prompt: at most; they are ragged above 8).  idle, done:
    shares of the requests that bring none, and that end (all their pages come back).  drop: drafted tokens that some others lose."""
    return {"op": "step", "R": R, "longest": longest, "new": new, "page": page, "idle": idle, "done": done, "drop": drop}


def _append(R, new, hkv, D, page, x="bf16", cache="bf16", fused=True, pad=0):
    """fused: keys and values are parts of the rows of one projection.  pad: rows behind the last token."""
    return {"op": "append", "R": R, "new": new, "hkv": hkv, "D": D, "page": page, "x": x, "cache": cache, "fused": fused, "pad": pad}


def _attention(op, R, longest, new, hq, hkv, D, page, cache="bf16", window=0, sinks=0, ragged=True, pad=0):
    """longest: tokens of the longest request, its `new` ones among them.  ragged: the other requests have fewer of both (of new ones above 8)."""
    return {"op": op, "R": R, "longest": longest, "new": new, "hq": hq, "hkv": hkv, "D": D, "page": page, "cache": cache, "window": window,
            "sinks": sinks, "ragged": ragged, "pad": pad}


def listed():
    cases = {
        # a decoding step of 64 sequences, some of them waiting or just ended
        "step_r64": _step(64, 4096, 1, 16, idle=0.1, done=0.05),
        # a step of 512 requests that admits prompts, with drafted tokens lost elsewhere
        "step_r512": _step(512, 8192, 96, 32, idle=0.2, done=0.1, drop=3),
        # one token of 64 sequences, from the fused projection
        "append_m64": _append(64, 1, 8, 128, 16),
        # prompts in fp32 from the layers into a quantised cache, heads of 64
        "append_m4000": _append(6, 900, 16, 64, 64, x="f32", cache="mxint8", pad=37),
        # one sequence of a thousand tokens: latency
        "decode_r1": _attention("decode", 1, 1021, 1, 32, 8, 128, 16),
        # a serving batch with lengths spread over a factor of four, groups of five heads
        "decode_r64": _attention("decode", 64, 8191, 1, 40, 8, 128, 16),
        # as many key heads as query heads, quantised cache
        "decode_r24_mx": _attention("decode", 24, 4099, 1, 40, 40, 128, 64, cache="mxint8"),
        # four drafted tokens of eight long sequences under a window, the first tokens kept
        "decode_r8_window": _attention("decode", 8, 32000, 4, 32, 8, 128, 16, window=4096, sinks=4),
        # three short prompts of odd lengths, heads of 64, a padded batch
        "prompt_m201": _attention("prompt", 3, 97, 97, 16, 4, 64, 16, pad=11),
        # the last chunk of a prompt behind what is cached already
        "prompt_m2048_chunk": _attention("prompt", 1, 12288, 2048, 40, 8, 128, 16),
        # long prompts of two requests under a window with first tokens kept, quantised cache
        "prompt_m8000_window": _attention("prompt", 2, 5000, 5000, 32, 32, 128, 64, cache="mxint8", window=1024, sinks=16),
        # one prompt of 8192 tokens
        "prompt_m8192": _attention("prompt", 1, 8192, 8192, 32, 8, 128, 64),
    }
    return [dict(c, name=n) for n, c in cases.items()]


def draw(rng):
    """One more case of the same ranges."""
    def log_uniform(lo, hi):
        return int(round(lo * (hi / lo) ** rng.random()))

    op = rng.choice(("step", "append", "decode", "decode", "prompt", "prompt"))
    page = rng.choice((16, 16, 32, 64, 128))
    if op == "step":
        return _step(log_uniform(1, 512), log_uniform(64, 32768), rng.choice((1, 1, 4, log_uniform(8, 256))), page, rng.choice((0.0, 0.2)),
                     rng.choice((0.0, 0.1)), rng.choice((0, 3)))
    heads = [(32, 8), (40, 8), (32, 32), (40, 40), (16, 2), (16, 4), (8, 1), (24, 8), (16, 1)]
    hq, hkv = rng.choice(heads)
    D = rng.choice((128, 128, 64))
    cache = rng.choice(("bf16", "bf16", "mxint8"))
    if op == "append":
        R = log_uniform(1, 256)
        new = rng.choice((1, 1, log_uniform(2, 2048)))
        return _append(R, max(1, min(new, 4096 // R)), hkv, D, page, rng.choice(("f32", "bf16", "bf16")), cache, rng.random() < 0.6,
                       rng.choice((0, 0, 13)))
    window, sinks = rng.choice(((0, 0), (0, 0), (log_uniform(16, 4096), 0), (log_uniform(64, 4096), rng.randint(1, 64))))
    ragged, pad = rng.random() < 0.7, rng.choice((0, 0, 5))
    if op == "decode":
        new = rng.choice((1, 1, 1, rng.randint(2, 8)))
        R = log_uniform(1, 256)
        longest = min(log_uniform(64, 32768), 60_000_000 // (R * hkv * D), 400_000_000 // (R * hq * new))
        return _attention("decode", R, max(longest, new), new, hq, hkv, D, page, cache, window, sinks, ragged, pad)
    R = rng.choice((1, 1, 2, 3, log_uniform(1, 8)))
    new = log_uniform(9, 8192 // R)
    longest = new + rng.choice((0, 0, log_uniform(16, 8192)))
    longest = max(new, min(longest, 2_000_000_000 // (R * hq * new), 60_000_000 // (R * hkv * D)))
    return _attention("prompt", R, longest, new, hq, hkv, D, page, cache, window, sinks, ragged, pad)


# ---- the requests of a case ------------------------------------------------------------------------------------------------------

def _spread(r):
    """Evenly spread over [0, 1), the first 1: the share of the longest that request r has."""
    return 1.0 - (r * 0.6180339887498949) % 1.0


def _requests(case):
    """(tokens before the step, new ones or minus those that go) of every request."""
    R, new = case["R"], case["new"]
    if case["op"] == "append":
        return [(7 * r % 300, max(1, round(new * (0.4 + 0.6 * _spread(r)))) if new > 8 else new) for r in range(R)]
    if case["op"] == "step":
        out = []
        for r in range(R):
            n = max(1, round(new * _spread(3 * r))) if new > 8 else new
            before = max(0, round(case["longest"] * (0.05 + 0.95 * _spread(r))) - n)
            lot = (r * 0.7548776662466927 + 0.1) % 1.0
            if lot < case["done"]:
                out.append((before, -before))
            elif lot < case["done"] + case["idle"]:
                out.append((before, -min(before, case["drop"])))
            else:
                out.append((0 if new > 8 and r % 2 else before, n))
        return out
    out = []
    for r in range(R):
        share = 0.25 + 0.75 * _spread(r) if case["ragged"] else 1.0
        total = max(1, round(case["longest"] * share))
        n = min(total, max(1, round(new * share)) if new > 8 else new)
        out.append((total - n, n))
    return out


def _rows(case):
    return sum(max(0, n) for _, n in _requests(case)) + case.get("pad", 0)


def _generator(seed, case):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 8 + ("step", "append", "decode", "prompt").index(case["op"]))
    return g


def _pages(tokens, page):
    return (tokens + page - 1) // page


def _tables(case, g):
    """The tables before the step and after it, and the ring of free pages, with the pages in any order."""
    page, requests = case["page"], _requests(case)
    before = torch.tensor([b for b, _ in requests], device=DEV)
    added = torch.tensor([n for _, n in requests], device=DEV)
    after = before + added
    most = max(max(b, b + n) for b, n in requests)
    width = _pages(most, page) + 2
    held = torch.maximum(_pages(before, page), _pages(after, page))
    n_pages = int(held.sum()) + 5
    ids = torch.randperm(n_pages, generator=g, device=DEV, dtype=torch.int32)
    # the pages that the requests hold, then those that they will take, in the order of the requests
    col = torch.arange(width, device=DEV)
    old, new = col < _pages(before, page)[:, None], (col >= _pages(before, page)[:, None]) & (col < _pages(after, page)[:, None])
    n_old, n_new = int(old.sum()), int(new.sum())
    tables = torch.full((case["R"], width), -1, dtype=torch.int32, device=DEV)
    tables[old] = ids[:n_old]
    later = tables.clone()
    later[new] = ids[n_old:n_old + n_new]
    # the ring: what is free starts somewhere in the middle and runs over its end
    head = n_pages // 2 + 3 * n_pages
    free = torch.full((n_pages,), -1, dtype=torch.int32, device=DEV)
    left = ids[n_old:]
    free[(head + torch.arange(len(left), device=DEV)) % n_pages] = left
    ring = torch.tensor([head, head + len(left)], device=DEV)
    return {"before": before.int(), "added": added.int(), "tables": tables, "later": later, "free": free, "ring": ring, "n_pages": n_pages}


def _slots(tables, before, added, rows, page):
    """Slot and position of every row (-1 behind the last one)."""
    grow = added.clamp(min=0).long()
    ends = grow.cumsum(0)
    row = torch.arange(rows, device=DEV)
    of = torch.searchsorted(ends, row, right=True).clamp(max=len(ends) - 1)
    pos = row - (ends - grow)[of] + before.long()[of]
    slot = tables[of, (pos // page).clamp(0, tables.shape[1] - 1)].long() * page + pos % page
    mine = row < ends[-1]
    return torch.where(mine, slot, -1).int(), torch.where(mine, pos, -1).int()


def _normal(shape, kind, g, spread=1.0):
    """Normal values with a few outlier channels."""
    x = torch.randn(shape, generator=g, device=DEV) * spread
    at = torch.randint(0, shape[-1], (max(1, shape[-1] // 64),), generator=g, device=DEV)
    x[..., at] *= 3.0
    return x.to(_FLOAT[kind])


def _inputs(case, seed):
    """What the program has in hand, as plain tensors."""
    g = _generator(seed, case)
    s = _tables(case, g)
    if case["op"] == "step":
        return s
    rows, hkv, D, page = _rows(case), case["hkv"], case["D"], case["page"]
    s["slots"], s["pos"] = _slots(s["later"], s["before"], s["added"], rows, page)
    shape = (s["n_pages"], hkv, page, D)
    for name in ("keys", "values"):
        x = _normal(shape, "bf16", g)
        s[name] = _pack(*_quantised(x.view(-1, D).double(), BITS)) if case["cache"] == "mxint8" else x
    if case["op"] == "append":
        if case["fused"]:
            hq = 4 * hkv
            both = _normal((rows, (hq + 2 * hkv) * D), case["x"], g)
            s["k"] = both[:, hq * D:(hq + hkv) * D].unflatten(1, (hkv, D))
            s["v"] = both[:, (hq + hkv) * D:].unflatten(1, (hkv, D))
        else:
            s["k"], s["v"] = _normal((rows, hkv, D), case["x"], g), _normal((rows, hkv, D), case["x"], g)
    else:
        s["q"] = _normal((rows, case["hq"], D), "bf16", g, 1.5)
        s["y"] = torch.zeros((rows, case["hq"], D), dtype=torch.bfloat16, device=DEV)
    return s


def prepare(case, seed):
    s = dict(_inputs(case, seed), case=dict(case), rows=_rows(case), most=max(b + n for b, n in _requests(case)),
             new=max(1, max(n for _, n in _requests(case))))
    if own:
        import paper_2402_02446_b200 as L
        pages = s["pages"] = L.new_page_table(case["R"], s["tables"].shape[1], s["n_pages"], case["page"])
        for mine, given in ((pages.tables, s["tables"]), (pages.free, s["free"]), (pages.ring, s["ring"]), (pages.lengths, s["before"])):
            mine.copy_(given)
        s["step"] = L.cache_step(pages, s["added"], s["rows"], max_added=s["new"], commit=False)
        if case["op"] != "step":
            s["cache"] = L.new_kv_cache(s["n_pages"], case["page"], case["hkv"], case["D"], dtype=L.MXINT8 if case["cache"] == "mxint8" else torch.bfloat16)
            s["cache"].keys.copy_(s["keys"])
            s["cache"].values.copy_(s["values"])
    return s


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- the calls of the library ----------------------------------------------------------------------------------------------------

def _run_own(s):
    import paper_2402_02446_b200 as L
    c = s["case"]
    if c["op"] == "step":
        step = L.cache_step(s["pages"], s["added"], s["rows"], max_added=s["new"], step=s["step"], commit=False)
        return {"tables": s["pages"].tables, "free": s["pages"].free, "slots": step.slots, "pos": step.positions, "lengths": step.lengths, "ring": step.ring}
    cache = s["cache"]
    if c["op"] == "append":
        L.append_kv(s["k"], s["v"], cache, s["step"].slots)
        if c["cache"] == "bf16":
            return {"keys": cache.keys, "values": cache.values}
        n = s["n_pages"] * c["hkv"] * c["page"]
        return {"keys": L.dequantize_activations(cache.keys, n, c["D"], out_dtype=torch.bfloat16),
                "values": L.dequantize_activations(cache.values, n, c["D"], out_dtype=torch.bfloat16)}
    return {"y": L.paged_attention(s["q"], cache, s["pages"], s["step"], window=c["window"], sinks=c["sinks"], Y=s["y"])}


# ---- the plain forms -------------------------------------------------------------------------------------------------------------

def _quantised(v, bits):
    """Mantissas and exponents (blocks of 16 along the row) of fp64 values."""
    b = v.unflatten(-1, (-1, BLOCK))
    e = (torch.frexp(b.abs().amax(-1, keepdim=True))[1] - 1).clamp(EXP_MIN, EXP_MAX)
    top = 2 ** (bits - 1) - 1
    m = torch.round(torch.ldexp(b, bits - 2 - e)).clamp(-top, top)
    return m.flatten(-2), e.squeeze(-1)


def _pack(m, e):
    """The library's MXINT8 buffer: mantissas, then exponent bytes."""
    return torch.cat([m.to(torch.int8).view(torch.uint8).flatten(), (e + 127).to(torch.uint8).flatten()])


def _unpacked(buf, rows, cols, dtype=torch.float32):
    m = buf[:rows * cols].view(torch.int8).view(rows, cols).to(dtype)
    e = buf[rows * cols:].view(rows, cols // BLOCK).int() - 127 - (BITS - 2)
    return (m.unflatten(-1, (-1, BLOCK)) * torch.ldexp(torch.ones_like(e, dtype=dtype), e)[..., None]).flatten(-2)


def _cache_values(s, name, dtype=torch.float32):
    """[pages, heads, page, D] in the given type."""
    c = s["case"]
    shape = (s["n_pages"], c["hkv"], c["page"], c["D"])
    if c["cache"] == "bf16":
        return s[name].to(dtype)
    return _unpacked(s[name], shape[0] * shape[1] * shape[2], shape[3], dtype).view(shape)


def _run_plain(s):
    c = s["case"]
    return {"step": _plain_step, "append": _plain_append}.get(c["op"], _plain_attention)(s, c)


def _plain_step(s, c):
    page, n = c["page"], s["n_pages"]
    before, lengths = s["before"].long(), (s["before"] + s["added"]).clamp(min=0).long()
    have, want = _pages(before, page)[:, None], _pages(lengths, page)[:, None]
    col = torch.arange(s["tables"].shape[1], device=DEV)
    head, tail = s["ring"][0], s["ring"][1]
    # the pages that go, to the ring's tail, and then those that are wanted, from its head, each in the order of the requests
    gone, fresh = ((col >= want) & (col < have)).flatten(), ((col >= have) & (col < want)).flatten()
    at = torch.where(gone, (tail + gone.cumsum(0) - 1) % n, n)
    free = torch.cat([s["free"], s["free"].new_zeros(1)]).scatter_(0, at, s["tables"].flatten())[:n]
    got = free[(head + fresh.cumsum(0) - 1) % n]
    tables = torch.where(fresh, got, s["tables"].flatten()).view(s["tables"].shape)
    slots, pos = _slots(tables, s["before"], s["added"], s["rows"], page)
    return {"tables": tables, "free": free, "slots": slots, "pos": pos, "lengths": lengths.int(), "ring": torch.stack([head + fresh.sum(), tail + gone.sum()])}


def _plain_append(s, c):
    page, hkv, D = c["page"], c["hkv"], c["D"]
    mine = s["slots"] >= 0
    at, off = s["slots"][mine].long() // page, s["slots"][mine].long() % page
    if c["cache"] == "bf16":
        s["keys"][at, :, off] = s["k"][mine].bfloat16()
        s["values"][at, :, off] = s["v"][mine].bfloat16()
        return {"keys": s["keys"], "values": s["values"]}
    n = s["n_pages"] * hkv * page
    return {"keys": _appended(s["keys"], s["k"][mine], at, off, n, c), "values": _appended(s["values"], s["v"][mine], at, off, n, c)}


def _appended(buf, x, at, off, n, c):
    """Rows into a quantised cache; all of it as values."""
    m, e = _quantised(x.double(), BITS)
    D, shape = c["D"], (-1, c["hkv"], c["page"])
    buf[:n * D].view(torch.int8).view(*shape, D)[at, :, off] = m.to(torch.int8)
    buf[n * D:].view(*shape, D // BLOCK)[at, :, off] = (e + 127).to(torch.uint8)
    return _unpacked(buf, n, D).bfloat16()


def _plain_attention(s, c):
    R, hq, hkv, D, page, L, n = c["R"], c["hq"], c["hkv"], c["D"], c["page"], s["most"], s["new"]
    group = hq // hkv
    ids = s["later"][:, :_pages(L, page)].clamp(min=0).long()
    k, v = (_cache_values(s, name)[ids].transpose(1, 2).flatten(2, 3)[:, :, :L] for name in ("keys", "values"))       # [R, hkv, L, D]
    row0 = s["added"].long().cumsum(0) - s["added"]
    i = torch.arange(n, device=DEV)
    row = (row0[:, None] + i).clamp(max=s["rows"] - 1)
    q = s["q"][row].float().view(R, n, hkv, group, D).permute(0, 2, 3, 1, 4).reshape(R, hkv, group * n, D)
    pos = (s["before"][:, None] + i)[:, :, None]                                                                      # [R, n, 1]
    j = torch.arange(L, device=DEV)
    seen = j <= pos
    if c["window"]:
        seen &= (j > pos - c["window"]) | (j < c["sinks"])
    p = torch.matmul(q, k.transpose(2, 3)).mul_(1.0 / math.sqrt(D)).view(R, hkv, group, n, L)
    p.masked_fill_(~seen[:, None, None], -math.inf)
    p.sub_(p.amax(-1, keepdim=True)).exp_()
    total = p.sum(-1, keepdim=True)
    y = torch.matmul(p.view(R, hkv, group * n, L), v).view(R, hkv, group, n, D).div_(total)
    y = y.permute(0, 3, 1, 2, 4).reshape(R, n, hq, D).bfloat16()
    mine = i < s["added"][:, None]
    s["y"][row[mine]] = y[mine]
    return {"y": s["y"]}


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------------------

def exact(case, seed):
    if case["op"] == "step":
        return None
    s = dict(_inputs(case, seed), case=case)
    requests, page, hkv, D = _requests(case), case["page"], case["hkv"], case["D"]
    slots = s["slots"].long()
    if case["op"] == "append":
        out = {}
        mine = (slots >= 0).nonzero()[:, 0]
        for name, x in (("keys", s["k"]), ("values", s["v"])):
            w = _cache_values(s, name, torch.float64)
            x = x[mine].double()
            if case["cache"] == "mxint8":
                b = x.unflatten(-1, (-1, BLOCK))
                power = torch.floor(torch.log2(b.abs().amax(-1)))
                grain = torch.pow(2.0, power.clamp(EXP_MIN, EXP_MAX) - (BITS - 2))[..., None]
                top = 2.0 ** (BITS - 1) - 1
                x = (torch.clamp(torch.round(b / grain), -top, top) * grain).flatten(-2)
            w[slots[mine] // page, :, slots[mine] % page] = x
            out[name] = w if case["cache"] == "bf16" else w.view(-1, D)
        return out
    y = torch.zeros((_rows(case), case["hq"], D), dtype=torch.float64, device=DEV)
    group, row = case["hq"] // hkv, 0
    for r, (before, n) in enumerate(requests):
        ids = s["later"][r, :_pages(before + n, page)].long()
        one = dict(s, keys=s["keys"], values=s["values"])
        k, v = (_request_values(one, case, name, ids)[:, :before + n] for name in ("keys", "values"))
        for h in range(hkv):
            for at in range(0, n, 1024):
                m = min(1024, n - at)
                q = s["q"][row + at:row + at + m, h * group:(h + 1) * group].double()
                pos = torch.arange(before + at, before + at + m, device=DEV)[:, None, None]
                j = torch.arange(before + n, device=DEV)
                hidden = j > pos
                if case["window"]:
                    hidden = hidden | ((pos - j >= case["window"]) & (j >= case["sinks"]))
                score = torch.einsum("mgd,ld->mgl", q, k[h]) / math.sqrt(D)
                y[row + at:row + at + m, h * group:(h + 1) * group] = torch.softmax(score.masked_fill(hidden, -math.inf), -1) @ v[h]
        row += n
    return {"y": y}


def _request_values(s, case, name, ids):
    """[heads, tokens, D] of a request's pages, in 64 bits."""
    hkv, page, D = case["hkv"], case["page"], case["D"]
    if case["cache"] == "bf16":
        x = s[name][ids].double()
    else:
        n = s["n_pages"] * hkv * page
        m = s[name][:n * D].view(torch.int8).view(-1, hkv, page, D)[ids].double()
        e = s[name][n * D:].view(-1, hkv, page, D // BLOCK)[ids].double()
        x = m * torch.pow(2.0, e - 127 - (BITS - 2)).repeat_interleave(BLOCK, -1)
    return x.transpose(0, 1).flatten(1, 2)


def _visible(case):
    """(pairs of a query and a key that it sees, keys that a request's queries see) over the requests."""
    pairs = keys = 0
    w, s = case["window"], case["sinks"]
    for before, n in _requests(case):
        total = before + n
        if not w:
            pairs += n * before + n * (n + 1) // 2
            keys += total
            continue
        first = max(0, before - w + 1)
        keys += total - first + min(s, first)
        pairs += sum(min(p + 1, w) + min(s, max(0, p + 1 - w)) for p in range(before, total))
    return pairs, keys


def work(case):
    requests = _requests(case)
    new = sum(max(0, n) for _, n in requests)
    if case["op"] == "step":
        page = case["page"]
        moved = sum(abs(_pages(b + n, page) - _pages(b, page)) for b, n in requests)
        # lengths and added in, lengths out, the pages that come or go (from one list, to the other), a row's page, slot and position
        return {"bytes": 12.0 * case["R"] + 8.0 * moved + 8.0 * new, "flops": 0.0}
    if case["op"] == "append":
        n = 2 * new * case["hkv"] * case["D"]
        return {"bytes": n * (_BYTES[case["x"]] + _BYTES[case["cache"]]) + 4.0 * new, "flops": 0.0}
    pairs, keys = _visible(case)
    return {"bytes": 2.0 * keys * case["hkv"] * case["D"] * _BYTES[case["cache"]] + 4.0 * new * case["hq"] * case["D"],
            "flops": 4.0 * pairs * case["hq"] * case["D"]}
