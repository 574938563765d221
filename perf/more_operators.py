"""A step's new rows, rotated to their positions, an 8-bit cache and attention over it, case by case.

A case is a dict of plain values.  `op` says what is called:

  rotate   pp_kv_rotate: norms of query and key heads and the rotation to their
           positions, keys and values straight into the paged cache or to rows
  write8   pp_kv_write8: the step's K and V rows into a cache of 8-bit numbers
           with a power-of-two scale for each block of tokens and head
  attend8  pp_paged_attention8: the step's new tokens over that cache, by chunks
           or by single tokens

Head layouts are those behind the synthetic workloads' KV bytes per token (16
query heads on 2, 28 on 4, plain multi-head) and odd ones.  Lengths, orders of
slots and head counts follow from the case alone (its `shape` number), values
from the seed.  Rows of an 8-bit cache that hold no token of a request are NaN,
and exponents of blocks that hold none are any number.
"""
import math
import random

import numpy as np
import torch

own = False

LEAST, MOST = -40, 40                       # exponents of a scale


def _rotate(name, tokens, heads, kv_heads, dim, rotated, layout, dtype, norm, to, block, longest, factor, original, shape):
    """rotated: elements of a head that turn; to: "cache" or "rows"; factor and original: scaling of the frequencies
    (original 0: all alike)."""
    return dict(name=name, op="rotate", tokens=tokens, heads=heads, kv_heads=kv_heads, dim=dim, rotated=rotated,
                layout=layout, dtype=dtype, norm=norm, to=to, block=block, longest=longest, factor=factor,
                original=original, shape=shape)


def _write8(name, tokens, run, kv_heads, dim, dtype, block, order, shape):
    """run: a request's new tokens, "lo-hi"."""
    return dict(name=name, op="write8", tokens=tokens, run=run, kv_heads=kv_heads, dim=dim, dtype=dtype, block=block,
                order=order, shape=shape)


def _attend8(name, requests, fresh, cached, heads, kv_heads, dim, dtype, block, shape, window=0, order="token"):
    """fresh and cached: the smallest and the largest count, "lo-hi"."""
    return dict(name=name, op="attend8", requests=requests, fresh=fresh, cached=cached, heads=heads,
                kv_heads=kv_heads, dim=dim, dtype=dtype, block=block, window=window, order=order, shape=shape)


def listed():
    return [
        # a decode step's rows: latency
        _rotate("rotate-decode", 64, 16, 2, 128, 128, "half", "bf16", True, "cache", 16, 16_000, 1.0, 0, 1),
        # an odd layout, part of each head turns, positions far beyond the original context, rows for another write
        _rotate("rotate-odd", 5003, 9, 3, 80, 32, "interleaved", "f16", False, "rows", 32, 1_000_000, 8.0, 0, 2),
        # a large prefill step with frequencies scaled by parts
        _rotate("rotate-prefill", 30_011, 28, 4, 128, 128, "half", "bf16", True, "cache", 16, 120_000, 4.0, 32_768, 3),
        # a decode step: a row more in each running request's last block
        _write8("write8-decode", 64, "1-1", 2, 128, "bf16", 16, "token", 4),
        # short chunks of an odd layout, heads outside tokens in the cache
        _write8("write8-odd", 5003, "1-150", 3, 80, "f16", 32, "head", 5),
        # the rows of a large prefill step
        _write8("write8-prefill", 30_011, "500-9000", 4, 128, "bf16", 16, "token", 6),
        # a few short requests decode: latency
        _attend8("attend8-few", 4, "1-1", "36-900", 16, 2, 128, "bf16", 16, 7),
        # a full decode batch of ragged lengths, seven query heads per K/V head
        _attend8("attend8-batch", 128, "1-1", "200-16000", 28, 4, 128, "bf16", 16, 8),
        # two very long contexts decode: rows are few, the split is along the context
        _attend8("attend8-long", 2, "1-1", "131000-200000", 16, 2, 128, "f16", 32, 9),
        # new turns after resident prefixes
        _attend8("chunk8-turns", 8, "60-700", "512-8192", 16, 2, 128, "bf16", 16, 10),
        # a ragged mixed step of a multi-head layout with a sliding window; one-token requests among long chunks
        _attend8("chunk8-ragged", 24, "1-2000", "0-6000", 16, 16, 64, "f16", 32, 11, window=1500, order="head"),
        # a long prompt's last large chunk
        _attend8("chunk8-large", 1, "8192-8192", "24576-24576", 28, 4, 128, "bf16", 64, 12),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    shape = rng.randrange(1 << 30)
    block = rng.choice([8, 16, 16, 32, 64, 128])
    op = rng.choice(["rotate", "rotate", "write8", "attend8", "attend8", "attend8"])
    order = rng.choice(["token", "head"])
    dtype = rng.choice(["bf16", "f16"])
    dim = rng.choice([64, 80, 96, 128, 128, 128])
    kv_heads = rng.choice([1, 2, 3, 4, 5, 8])
    group = rng.choice([1, 2, 4, 7, 8])
    if op == "rotate":
        tokens = _log_int(rng, 1, 30_011 * 28 // max(28, kv_heads * group))
        rotated = rng.choice([dim, dim, dim // 2, dim // 4])
        factor = rng.choice([1.0, 1.0, 4.0, 8.0, 32.0])
        return _rotate("", tokens, kv_heads * group, kv_heads, dim, rotated, rng.choice(["half", "half", "interleaved"]),
                       dtype, rng.random() < 0.6, rng.choice(["cache", "rows"]), block, _log_int(rng, 100, 2_000_000),
                       factor, rng.choice([0, 8192, 32_768]) if factor > 1 else 0, shape)
    if op == "write8":
        tokens = _log_int(rng, 1, 30_011 * 4 // max(4, kv_heads))
        longest = _log_int(rng, 1, 9000)
        return _write8("", tokens, f"{rng.choice([1, (longest + 1) // 2])}-{longest}", kv_heads, dim, dtype, block, order, shape)
    window = rng.choice([0, 0, 0, _log_int(rng, 50, 4000)])
    if rng.random() < 0.5:                  # single tokens
        requests = _log_int(rng, 1, 128)
        top = _log_int(rng, 100, min(200_000, 2_000_000 // (requests * kv_heads)))
        return _attend8("", requests, "1-1", f"{rng.randrange(top)}-{top}", kv_heads * group, kv_heads, dim, dtype,
                        block, shape, window, order)
    requests = _log_int(rng, 1, 24)
    fresh = _log_int(rng, 2, 8192 // requests)
    cached = _log_int(rng, 1, 24_000 // requests)
    low = rng.choice([0, 1, fresh])
    return _attend8("", requests, f"{low}-{fresh}", f"{rng.choice([0, cached])}-{cached}", kv_heads * group, kv_heads,
                    dim, dtype, block, shape, window, order)


# ---------------------------------------------------------------------------
# Shapes: what follows from the case alone.
# ---------------------------------------------------------------------------
def _lengths(requests, fresh, cached, shape):
    """Per request: new tokens and tokens in the cache, over the whole range."""
    rng = random.Random(shape)
    f_lo, f_hi = (int(x) for x in fresh.split("-"))
    c_lo, c_hi = (int(x) for x in cached.split("-"))
    out = []
    for r in range(requests):
        f = f_lo + int(round((f_hi - f_lo) * rng.random() ** 2))
        c = c_lo + int(round((c_hi - c_lo) * rng.random() ** 2))
        out.append((f_hi if r == 0 else f, c_hi if r == requests - 1 else c))
    return out


def _runs(case):
    """Per request: the place in its block where its new rows begin, and their count; tokens in all."""
    rng = random.Random(case["shape"])
    lo, hi = (int(x) for x in case["run"].split("-"))
    out, left = [], case["tokens"]
    while left > 0:
        n = min(left, rng.randint(lo, hi))
        out.append((rng.randrange(case["block"]) if rng.random() < 0.7 else 0, n))
        left -= n
    return out


def _touched(case):
    """Blocks that the new rows are in."""
    return sum((first + n - 1) // case["block"] + 1 for first, n in _runs(case))


def _pairs(fresh, cached, window):
    """Visible (query, key) pairs of one request."""
    pos = np.arange(cached, cached + fresh, dtype=np.int64) + 1
    return int(np.minimum(pos, window).sum() if window else pos.sum())


def work(case):
    row = case["kv_heads"] * case["dim"]
    if case["op"] == "rotate":
        turned = (case["heads"] + case["kv_heads"]) * case["dim"] * case["tokens"]
        rows = turned + (row * case["tokens"] if case["to"] == "cache" else 0)
        return {"bytes": 4 * rows + (12 if case["to"] == "cache" else 4) * case["tokens"],
                "flops": turned * (7 if case["norm"] else 3)}
    if case["op"] == "write8":
        # rows of 16 bits in, of 8 bits out; a slot a token; exponents read and written
        return {"bytes": case["tokens"] * (6 * row + 8) + 4 * _touched(case) * case["kv_heads"],
                "flops": 4 * case["tokens"] * row}
    lens = _lengths(case["requests"], case["fresh"], case["cached"], case["shape"])
    window = case["window"]
    pairs = sum(_pairs(f, c, window) for f, c in lens)
    keys = sum((min(f + c, f + window - 1) if window else f + c) for f, c in lens if f)
    tokens = sum(f for f, _ in lens)
    blocks = sum(-(-(f + c) // case["block"]) for f, c in lens)
    return {"bytes": 2 * row * keys + 4 * tokens * case["heads"] * case["dim"] + 4 * tokens * case["heads"]
            + (4 + 2 * case["kv_heads"]) * blocks,
            "flops": 4 * case["dim"] * case["heads"] * pairs}


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float16


def _cache(case, blocks, gen):
    """[blocks][block][kv_heads][dim], tokens outside heads or (a view) heads outside tokens."""
    b, h, d = case["block"], case["kv_heads"], case["dim"]
    shape = (blocks, b, h, d) if case.get("order", "token") == "token" else (blocks, h, b, d)
    t = torch.empty(shape, dtype=_dtype(case), device="cuda").normal_(generator=gen)
    return t if case.get("order", "token") == "token" else t.transpose(1, 2)


def _to8(cache):
    """A cache of any numbers as 8-bit numbers (same order of dimensions) and exponents [blocks][heads]."""
    top = cache.float().abs().amax((1, 3))
    fraction, power = torch.frexp(top)
    e = (power - 9 + (fraction > 0.875)).clamp(LEAST, MOST)
    code = torch.ldexp(cache.float(), -e[:, None, :, None]).to(torch.float8_e4m3fn)
    return code, e.to(torch.int8)


def _handle(cache, case):
    if not own:
        return None
    from paper_2608_01655_gb300 import binding as pp
    return pp.KVCache.like(cache, dtype=_dtype(case))


def _i32(a):
    return torch.tensor(np.asarray(a, np.int32), device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    rng = np.random.default_rng(seed)
    return {"rotate": _prepare_rotate, "write8": _prepare_write8, "attend8": _prepare_attend8}[case["op"]](case, gen, rng)


SLOW, FAST, BASE = 1.0, 32.0, 10_000.0


def _frequencies(case):
    """Radians a token of each pair, in 64 bits."""
    r = case["rotated"]
    f = BASE ** (-np.arange(0, r, 2, dtype=np.float64) / r)
    if not case["original"]:
        return f / case["factor"]
    turns = case["original"] * f / (2 * math.pi)
    keep = np.clip((turns - SLOW) / (FAST - SLOW), 0, 1)
    return f * (keep + (1 - keep) / case["factor"])


def _amplitude(case):
    return 1.0 if not case["original"] else 0.1 * math.log(case["factor"]) + 1.0


def _rotary(case):
    """What a program keeps for the rotation."""
    if own:
        from paper_2608_01655_gb300 import binding as pp
        return pp.Rotary(case["rotated"], base=BASE, factor=case["factor"], original=case["original"], slow=SLOW,
                         fast=FAST, amplitude=_amplitude(case), interleaved=case["layout"] == "interleaved")
    return torch.tensor(_frequencies(case), device="cuda")


def _prepare_rotate(case, gen, rng):
    tokens, hq, h, d = case["tokens"], case["heads"], case["kv_heads"], case["dim"]
    dtype = _dtype(case)
    # queries, keys and values are slices of the projection's output
    qkv = torch.empty((tokens, (hq + 2 * h) * d), dtype=dtype, device="cuda").normal_(generator=gen).mul_(2)
    q, k, v = (x.unflatten(1, (-1, d)) for x in qkv.split((hq * d, h * d, h * d), 1))
    weight = lambda: (torch.randn(d, generator=gen, device="cuda") * 0.2 + 1).to(dtype) if case["norm"] else None
    shape = random.Random(case["shape"])
    # runs of neighbouring positions (chunks) or single ones
    position = np.zeros(tokens, np.int64)
    at = 0
    while at < tokens:
        n = 1 if tokens <= 128 else shape.randint(1, 4000)
        first = shape.randrange(case["longest"])
        position[at:at + n] = first + np.arange(len(position[at:at + n]))
        at += n
    state = dict(case=case, q=q, k=k, v=v, q_weight=weight(), k_weight=weight(), rotary=_rotary(case),
                 position=_i32(position + rng.integers(0, 64)), q_out=torch.empty((tokens, hq, d), dtype=dtype, device="cuda"))
    blocks = -(-tokens * 5 // 4 // case["block"]) + 2 if case["to"] == "cache" else 1
    state.update(kc=_cache(case, blocks, gen), vc=_cache(case, blocks, gen))
    state["kv"] = _handle(state["kc"], case)
    if case["to"] == "rows":
        state["k_out"] = torch.empty((tokens, h, d), dtype=dtype, device="cuda")
    else:
        order = torch.randperm(blocks, generator=gen, device="cuda")
        slot = (order[:, None] * case["block"] + torch.arange(case["block"], device="cuda")).flatten()
        slot = slot[5:5 + tokens].contiguous()
        slot[torch.arange(tokens, device="cuda") % 37 == 36] = -1         # some tokens are padding
        state["slot"] = slot
    return state


def _prepare_write8(case, gen, rng):
    tokens, h, d, block = case["tokens"], case["kv_heads"], case["dim"], case["block"]
    runs = _runs(case)
    runs = [runs[i] for i in rng.permutation(len(runs))]
    blocks = _touched(case) + 3
    order = rng.permutation(blocks)
    slot, at = [], 0
    for first, n in runs:
        place = first + np.arange(n)
        slot.append(order[at + place // block] * block + place % block)
        at += (first + n - 1) // block + 1
    slot = np.concatenate(slot)
    slot[np.arange(tokens) % 211 == 210] = -1                             # some tokens are padding
    # values of a channel keep their size, some channels are large; K and V are slices of the projection's output
    size = torch.exp(torch.randn((3, h, d), generator=gen, device="cuda"))
    qkv = torch.empty((tokens, 3, h, d), dtype=torch.float32, device="cuda").normal_(generator=gen).mul_(size).to(_dtype(case))
    old = [_to8((_cache(case, blocks, gen).float() * size[i + 1]).to(_dtype(case))) for i in range(2)]
    return dict(case=case, kv=_handle(old[0][0], case), k=qkv[:, 1], v=qkv[:, 2], slot=torch.tensor(slot, device="cuda"),
                kc=old[0][0], ke=old[0][1], vc=old[1][0], ve=old[1][1])


def _prepare_attend8(case, gen, rng):
    lens = _lengths(case["requests"], case["fresh"], case["cached"], case["shape"])
    lens = [lens[i] for i in rng.permutation(len(lens))]
    block, h, d = case["block"], case["kv_heads"], case["dim"]
    fresh = [f for f, _ in lens]
    length = [f + c for f, c in lens]
    need = [-(-n // block) for n in length]
    blocks = sum(need) + 5
    kc, vc = _cache(case, blocks, gen), _cache(case, blocks, gen)
    # keys share a direction and queries are long: softmax weights are spread over decades; blocks differ in size
    kc += torch.randn((h, d), generator=gen, device="cuda").to(kc.dtype) * 0.5
    vc *= torch.exp(torch.randn((blocks, 1, h, 1), generator=gen, device="cuda")).to(vc.dtype)
    (kc, ke), (vc, ve) = _to8(kc), _to8(vc)
    order = rng.permutation(blocks)
    width = max(need) + 1
    table = np.full((len(lens), width), -1)
    at, empty = 0, []
    for r, n in enumerate(need):
        table[r, :n] = order[at:at + n]
        at += n
        if length[r] % block:
            empty.append(order[at - 1] * block + np.arange(length[r] % block, block))
    empty.append((order[at:, None] * block + np.arange(block)).reshape(-1))
    empty = torch.tensor(np.concatenate(empty), device="cuda")
    for c in (kc, vc):
        c.view(torch.uint8)[empty // block, empty % block] = 0x7f         # NaN
    unused = torch.tensor(order[at:], device="cuda")
    ke[unused], ve[unused] = 127, -128
    tokens = sum(fresh)
    # the queries are a slice of the projection's output
    qkv = torch.empty((tokens, (case["heads"] + 2 * h) * d), dtype=_dtype(case), device="cuda")
    qkv = qkv.normal_(generator=gen).mul_(2)
    q = qkv[:, :case["heads"] * d].unflatten(1, (case["heads"], d))
    kv, workspace = _handle(kc, case), None
    if own:
        workspace = torch.empty(kv.workspace_size(len(lens), width, sum(need)), dtype=torch.uint8, device="cuda")
    return dict(case=case, kv=kv, workspace=workspace, q=q, kc=kc, ke=ke, vc=vc, ve=ve, table=_i32(table),
                q_start=_i32(np.concatenate([[0], np.cumsum(fresh)])), length=_i32(length),
                fresh_host=fresh, length_host=length, max_q=max(fresh), scale=d ** -0.5,
                out=torch.empty((tokens, case["heads"], d), dtype=q.dtype, device="cuda"),
                lse=torch.empty((tokens, case["heads"]), dtype=torch.float32, device="cuda"))


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------
def run(state):
    op = state["case"]["op"]
    if own:
        from paper_2608_01655_gb300 import binding as pp
        return {"rotate": _own_rotate, "write8": _own_write8, "attend8": _own_attend8}[op](pp, state)
    return {"rotate": _plain_rotate, "write8": _plain_write8, "attend8": _plain_attend8}[op](state)


EPS = 1e-6


def _own_rotate(pp, s):
    if s["case"]["to"] == "rows":
        pp.pp_kv_rotate(s["kv"], s["rotary"], s["q"], s["k"], s["position"], s["q_out"], k_out=s["k_out"],
                        q_weight=s["q_weight"], k_weight=s["k_weight"], eps=EPS)
        return {"q": s["q_out"], "k": s["k_out"]}
    pp.pp_kv_rotate(s["kv"], s["rotary"], s["q"], s["k"], s["position"], s["q_out"], q_weight=s["q_weight"],
                    k_weight=s["k_weight"], eps=EPS, v=s["v"], slot_map=s["slot"], k_cache=s["kc"], v_cache=s["vc"])
    return {"q": s["q_out"], "kc": s["kc"], "vc": s["vc"]}


def _own_write8(pp, s):
    pp.pp_kv_write8(s["kv"], s["k"], s["v"], s["slot"], s["kc"], s["ke"], s["vc"], s["ve"])
    return {key: s[key] for key in ("kc", "ke", "vc", "ve")}


def _own_attend8(pp, s):
    pp.pp_paged_attention8(s["kv"], s["q"], s["kc"], s["ke"], s["vc"], s["ve"], s["table"], s["q_start"], s["length"],
                           s["max_q"], s["out"], s["scale"], window=s["case"]["window"], lse=s["lse"],
                           workspace=s["workspace"])
    return {"out": s["out"], "lse": s["lse"]}


def _plain_turn(x, weight, cos, sin, rotated, interleaved):
    """Rows [T][heads][dim] of one kind, in 32 bits."""
    y = x.float()
    if weight is not None:
        y = y * (y.square().mean(-1, keepdim=True) + EPS).rsqrt() * weight.float()
    a, b = (y[..., 0:rotated:2], y[..., 1:rotated:2]) if interleaved else (y[..., :rotated // 2], y[..., rotated // 2:rotated])
    low, high = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack((low, high), -1).flatten(-2) if interleaved else torch.cat((low, high), -1)
    return torch.cat((turned, y[..., rotated:]), -1).to(x.dtype)


def _plain_rotate(s):
    case = s["case"]
    angle = s["position"].double()[:, None, None] * s["rotary"]
    cos, sin = (f(angle).mul_(_amplitude(case)).float() for f in (torch.cos, torch.sin))
    inter = case["layout"] == "interleaved"
    q = _plain_turn(s["q"], s["q_weight"], cos, sin, case["rotated"], inter)
    k = _plain_turn(s["k"], s["k_weight"], cos, sin, case["rotated"], inter)
    if case["to"] == "rows":
        return {"q": q, "k": k}
    rows = (s["slot"] >= 0).nonzero()[:, 0]
    slot, block = s["slot"][rows], case["block"]
    s["kc"][slot // block, slot % block] = k[rows]
    s["vc"][slot // block, slot % block] = s["v"][rows]
    return {"q": q, "kc": s["kc"], "vc": s["vc"]}


def _plain_store8(x, cache, exponent, slot, block):
    """New rows [n][heads][dim] of finite numbers at slots, into codes and exponents."""
    where, which = torch.unique(slot // block, return_inverse=True)
    x = x.float()
    heads = x.shape[1]
    top = torch.zeros((len(where), heads), device=x.device)
    top.scatter_reduce_(0, which[:, None].expand(-1, heads), x.abs().amax(-1), "amax")
    fraction, power = torch.frexp(top)
    need = torch.where(top > 0, power - 9 + (fraction > 0.875), LEAST).clamp(LEAST, MOST)
    begun = torch.zeros(len(where), dtype=torch.bool, device=x.device)
    begun[which[slot % block == 0]] = True
    old = exponent[where].int()
    new = torch.where(begun[:, None], need, torch.maximum(old, need))
    down = torch.where(begun[:, None], 0, old - new)[:, None, :, None]
    raw = cache.view(torch.uint8)
    rows = torch.ldexp(raw[where].view(torch.float8_e4m3fn).float(), down)
    rows[which, slot % block] = torch.ldexp(x, -new[which][..., None]).clamp(-448, 448)
    raw[where] = rows.to(torch.float8_e4m3fn).view(torch.uint8)
    exponent[where] = new.to(torch.int8)


def _plain_write8(s):
    rows = (s["slot"] >= 0).nonzero()[:, 0]
    slot, block = s["slot"][rows], s["case"]["block"]
    _plain_store8(s["k"][rows], s["kc"], s["ke"], slot, block)
    _plain_store8(s["v"][rows], s["vc"], s["ve"], slot, block)
    return {key: s[key] for key in ("kc", "ke", "vc", "ve")}


def _plain_attend8(s):
    case = s["case"]
    group, window = case["heads"] // case["kv_heads"], case["window"]
    out, lse = torch.empty_like(s["out"]), torch.empty_like(s["lse"])
    at = 0
    for r, (fresh, n) in enumerate(zip(s["fresh_host"], s["length_host"])):
        if not fresh:
            continue
        ids = s["table"][r, :-(-n // case["block"])].long()
        k, v = (torch.ldexp(c.view(torch.uint8)[ids].view(torch.float8_e4m3fn).float(), e[ids].int()[:, None, :, None])
                .flatten(0, 1)[:n] for c, e in ((s["kc"], s["ke"]), (s["vc"], s["ve"])))
        k, v = k.permute(1, 2, 0), v.transpose(0, 1)                            # [h][d][n], [h][n][d]
        step = max(1, min(fresh, (1 << 29) // (n * case["heads"])))
        for a in range(0, fresh, step):
            b = min(fresh, a + step)
            q = s["q"][at + a:at + b].float().unflatten(1, (-1, group)).permute(1, 0, 2, 3)
            score = torch.matmul(q.flatten(1, 2), k).mul_(s["scale"]).unflatten(1, (b - a, group))
            if fresh > 1 or window:
                i = torch.arange(n - fresh + a, n - fresh + b, device=k.device)[:, None, None]
                j = torch.arange(n, device=k.device)
                score.masked_fill_((j > i) | (j <= i - window) if window else j > i, -math.inf)
            top = score.amax(-1, keepdim=True)
            p = score.sub_(top).exp_()
            total = p.sum(-1, keepdim=True)
            o = torch.matmul(p.flatten(1, 2), v).unflatten(1, (b - a, group)) / total
            out[at + a:at + b] = o.permute(1, 0, 2, 3).flatten(1, 2).to(out.dtype)
            lse[at + a:at + b] = (top + total.log())[..., 0].permute(1, 0, 2).flatten(1, 2)
        at += fresh
    return {"out": out, "lse": lse}


# ---------------------------------------------------------------------------
# The definition in 64 bits
# ---------------------------------------------------------------------------
def exact(case, seed):
    state = prepare(case, seed)
    return {"rotate": _exact_rotate, "write8": _exact_write8, "attend8": _exact_attend8}[case["op"]](case, state)


def _exact_rotate(case, s):
    """Pairs as complex numbers, times e^(i angle)."""
    r, half = case["rotated"], case["rotated"] // 2
    angle = s["position"].double()[:, None] * torch.tensor(_frequencies(case), device="cuda")
    spin = torch.polar(torch.full_like(angle, _amplitude(case)), angle)[:, None]
    out = {}
    for name in ("q", "k"):
        y = s[name].double()
        if case["norm"]:
            y = y / torch.sqrt((y * y).sum(-1, keepdim=True) / case["dim"] + EPS) * s[name + "_weight"].double()
        first = torch.arange(0, r, 2, device="cuda") if case["layout"] == "interleaved" else torch.arange(half, device="cuda")
        second = first + (1 if case["layout"] == "interleaved" else half)
        z = torch.complex(y[..., first], y[..., second]) * spin
        y[..., first], y[..., second] = z.real, z.imag
        out[name] = y
    if case["to"] == "rows":
        return out
    kc, vc = s["kc"].double(), s["vc"].double()
    slot = s["slot"].cpu().numpy()
    rows = np.flatnonzero(slot >= 0)
    where = (torch.tensor(slot[rows] // case["block"], device="cuda"), torch.tensor(slot[rows] % case["block"], device="cuda"))
    rows = torch.tensor(rows, device="cuda")
    return {"q": out["q"], "kc": kc.index_put(where, out["k"][rows]), "vc": vc.index_put(where, s["v"].double()[rows])}


def _exact_e4m3(y):
    """The nearest number of 4 significant bits, exponents from -6 on, ties to even."""
    size = torch.where(y == 0, 1, y.abs())
    step = torch.exp2(torch.floor(torch.log2(size)).clamp(min=-6) - 3)
    return (torch.round(y / step) * step).clamp(-448, 448)


def _exact_write8(case, s):
    """Block after block of all the cache; codes and exponents."""
    block = case["block"]
    slot = s["slot"].cpu().numpy()
    kept = np.flatnonzero(slot >= 0)
    token = np.full(s["kc"].shape[0] * block, -1)
    token[slot[kept]] = kept
    token = torch.tensor(token.reshape(-1, block), device="cuda")
    written, begun = token >= 0, (token[:, 0] >= 0)[:, None]
    out = {}
    for x, code, e in (("k", "kc", "ke"), ("v", "vc", "ve")):
        rows = torch.where(written[..., None, None], s[x].double()[token.clamp(min=0)], 0)      # [blocks][block][h][d]
        top = rows.abs().amax((1, 3))
        need = torch.full(top.shape, LEAST, device="cuda")
        for c in range(LEAST, MOST):
            need += top > 448 * 2.0 ** c
        old = s[e].long()
        any_row = written.any(1, keepdim=True)
        new = torch.where(any_row, torch.where(begun, need, torch.maximum(need, old)), old)
        down = torch.where(begun, 0, old - new)
        value = s[code].double() * torch.exp2(down.double())[:, None, :, None]
        value = torch.where(written[..., None, None], rows * torch.exp2(-new.double())[:, None, :, None], value)
        out[code], out[e] = _exact_e4m3(value), new
    return out


def _exact_attend8(case, s):
    block, group, window = case["block"], case["heads"] // case["kv_heads"], case["window"]
    out = torch.empty(s["out"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(s["lse"].shape, dtype=torch.float64, device="cuda")
    start = 0
    for r, (fresh, n) in enumerate(zip(s["fresh_host"], s["length_host"])):
        j = torch.arange(n, device="cuda")
        page = s["table"][r].long()[j // block]
        for h in range(case["kv_heads"]):
            k, v = (c.view(torch.uint8)[page, j % block, h].view(torch.float8_e4m3fn).double()
                    * torch.exp2(e[page, h].double())[:, None] for c, e in ((s["kc"], s["ke"]), (s["vc"], s["ve"])))
            for a in range(0, fresh, 1024):
                b = min(fresh, a + 1024)
                p = torch.arange(n - fresh + a, n - fresh + b, device="cuda")[:, None]
                seen = j[None] <= p
                if window:
                    seen &= j[None] > p - window
                for g in range(h * group, (h + 1) * group):
                    rows = slice(start + a, start + b)
                    x = (s["q"][rows, g].double() @ k.T) * s["scale"]
                    x = torch.where(seen, x, -math.inf)
                    lse[rows, g] = torch.logsumexp(x, 1)
                    out[rows, g] = torch.exp(x - lse[rows, g][:, None]) @ v
        start += fresh
    return {"out": out, "lse": lse}
