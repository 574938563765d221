"""Serving from a planned target: block tables, cache writes and paged attention, case by case.

A case is a dict of plain values.  `op` says what is called:

  tables   pp_block_tables: a step's block tables, slot map, positions and
           query offsets from the requests' lengths, with prefixes taken from
           the resident chunks of a prefix tree
  write    pp_kv_write: the step's new K and V rows into the paged cache
  attend   pp_paged_attention: the step's new tokens over the paged cache, by
           chunks or by single tokens

Chunks are 512 tokens as in the synthetic workloads; head layouts are those
behind their KV bytes per token (16 query heads on 2, 28 on 4, plain multi-head)
and odd ones.  Lengths, trees and head counts follow from the case alone (its
`shape` number), values and orders from the seed.  Rows of the cache that hold
no token of a request are NaN, as memory that nothing has written may be.
"""
import functools
import math
import random

import numpy as np
import torch

own = False

CHUNK_TOKENS = 512


def _tables(name, requests, admitted, chunks, depth, block, longest, shape):
    return dict(name=name, op="tables", requests=requests, admitted=admitted, chunks=chunks, depth=depth,
                block=block, longest=longest, shape=shape)


def _write(name, tokens, kv_heads, dim, dtype, block, order, shape):
    return dict(name=name, op="write", tokens=tokens, kv_heads=kv_heads, dim=dim, dtype=dtype, block=block,
                order=order, shape=shape)


def _attend(name, requests, fresh, cached, heads, kv_heads, dim, dtype, block, shape, window=0, order="token"):
    """fresh and cached: the smallest and the largest count, "lo-hi"."""
    return dict(name=name, op="attend", requests=requests, fresh=fresh, cached=cached, heads=heads,
                kv_heads=kv_heads, dim=dim, dtype=dtype, block=block, window=window, order=order, shape=shape)


def listed():
    return [
        # a small decode step: every running request gains one token
        _tables("tables-decode", 16, 0, 64, 8, 16, 2000, 1),
        # a burst of admissions: prompts that end in chunks of the tree, with tails of their own
        _tables("tables-admit", 192, 192, 10_000, 24, 16, 600, 2),
        # a large mixed step: a quarter admitted, long conversation chains, larger blocks
        _tables("tables-large", 2048, 512, 50_000, 64, 32, 9000, 3),
        # a decode step's rows
        _write("write-decode", 64, 2, 128, "bf16", 16, "token", 4),
        # odd head count and width, heads outside tokens in the cache
        _write("write-odd", 5003, 3, 80, "f16", 32, "head", 5),
        # the rows of a large prefill step
        _write("write-prefill", 30_011, 4, 128, "bf16", 16, "token", 6),
        # a few short requests decode: latency
        _attend("attend-few", 4, "1-1", "36-900", 16, 2, 128, "bf16", 16, 7),
        # a full decode batch of ragged lengths, seven query heads per K/V head
        _attend("attend-batch", 128, "1-1", "200-16000", 28, 4, 128, "bf16", 16, 8),
        # two very long contexts decode: rows are few, the split is along the context
        _attend("attend-long", 2, "1-1", "131000-200000", 16, 2, 128, "f16", 32, 9),
        # new turns after resident prefixes
        _attend("chunk-turns", 8, "60-700", "512-8192", 16, 2, 128, "bf16", 16, 10),
        # a ragged mixed step of a multi-head layout with a sliding window; one-token requests among long chunks
        _attend("chunk-ragged", 24, "1-2000", "0-6000", 16, 16, 64, "f16", 32, 11, window=1500, order="head"),
        # a long prompt's last large chunk
        _attend("chunk-large", 1, "8192-8192", "24576-24576", 28, 4, 128, "bf16", 64, 12),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    shape = rng.randrange(1 << 30)
    block = rng.choice([16, 16, 32, 64])
    op = rng.choice(["tables", "write", "attend", "attend"])
    if op == "tables":
        requests = _log_int(rng, 1, 2048)
        return _tables("", requests, rng.choice([0, requests // 3, requests]), _log_int(rng, 50, 50_000),
                       _log_int(rng, 2, 64), block, _log_int(rng, 20, 9000 if requests < 1000 else 2000), shape)
    order = rng.choice(["token", "head"])
    dtype = rng.choice(["bf16", "f16"])
    dim = rng.choice([64, 80, 96, 128, 128, 128])
    if op == "write":
        kv_heads = rng.choice([1, 2, 3, 4, 8])
        return _write("", _log_int(rng, 1, 30_011), kv_heads, dim, dtype, block, order, shape)
    kv_heads = rng.choice([1, 2, 4, 5, 8])
    group = rng.choice([1, 2, 4, 7, 8])
    heads = kv_heads * group
    window = rng.choice([0, 0, 0, _log_int(rng, 50, 4000)])
    if rng.random() < 0.5:                  # single tokens
        requests = _log_int(rng, 1, 128)
        top = _log_int(rng, 100, min(200_000, 2_000_000 // (requests * kv_heads)))
        return _attend("", requests, "1-1", f"{rng.randrange(top)}-{top}", heads, kv_heads, dim, dtype, block,
                       shape, window, order)
    requests = _log_int(rng, 1, 24)
    fresh = _log_int(rng, 2, 8192 // requests)
    cached = _log_int(rng, 1, 24_000 // requests)
    low = rng.choice([0, 1, fresh])
    return _attend("", requests, f"{low}-{fresh}", f"{rng.choice([0, cached])}-{cached}", heads, kv_heads, dim,
                   dtype, block, shape, window, order)


# ---------------------------------------------------------------------------
# Shapes: what follows from the case alone.
# ---------------------------------------------------------------------------
@functools.lru_cache(maxsize=8)
def _tree(chunks, depth, shape):
    """A prefix tree with a parent-closed resident set, laid out as blocks of a
    worker's cache: per chunk {up, base, begin, end}.  A run of chunks that
    follow one another down the tree and in the cache is one segment: `base` is
    the block at table index `begin`, `end` the table index after the chunk's
    last block and `up` the chunk above the segment.  A chunk that is not
    resident has base -1 and `up` its deepest resident ancestor."""
    rng = random.Random(shape)
    parent, level = [-1], [1]
    for i in range(1, chunks):
        p = i - 1 if rng.random() < 0.8 else rng.randrange(-1, i)
        if p >= 0 and level[p] >= depth:
            p = -1
        parent.append(p)
        level.append(1 if p < 0 else level[p] + 1)
    resident = [False] * chunks
    for i, p in enumerate(parent):
        resident[i] = (p < 0 or resident[p]) and rng.random() < 0.95
    size = [1] * chunks
    heavy = [-1] * chunks
    for i in range(chunks - 1, -1, -1):
        p = parent[i]
        if p >= 0 and resident[i]:
            size[p] += size[i]
    for i in range(chunks - 1, -1, -1):
        p = parent[i]
        if p >= 0 and resident[i] and (heavy[p] < 0 or size[i] >= size[heavy[p]]):
            heavy[p] = i
    unit = [[-1, -1, 0, 0] for _ in range(chunks)]      # in chunks, not in blocks
    used = 0
    for i, p in enumerate(parent):
        if not resident[i]:
            unit[i][0] = -1 if p < 0 else (p if resident[p] else unit[p][0])
        elif p < 0 or heavy[p] != i:                    # a segment's head: lay out the run below it
            begin, base, b = level[i] - 1, used, i
            while b >= 0:
                unit[b] = [p, base, begin, level[b]]
                used += 1
                b = heavy[b]
    hops = [0] * chunks
    for i in range(chunks):
        up = unit[i][0]
        hops[i] = 1 + (hops[up] if up >= 0 else 0)
    return np.array(parent, np.int32), np.array(unit, np.int32), used, max(hops)


@functools.lru_cache(maxsize=8)
def _table_shape(requests, admitted, chunks, depth, block, longest, shape):
    """Per request: node (-1: running already), length, tokens in the cache."""
    rng = random.Random(shape + 1)
    _, unit, _, _ = _tree(chunks, depth, shape)
    rows = []
    for r in range(requests):
        if r < admitted:
            node = rng.randrange(chunks)
            up = node if unit[node, 1] >= 0 else int(unit[node, 0])
            resident = int(unit[up, 3]) * CHUNK_TOKENS if up >= 0 else 0
            length = resident + rng.randrange(0 if resident else 1, longest + 1)
            cached = min(resident, max(length - 1, 0) // block * block)
            rows.append((node, length, cached))
        else:
            length = rng.randrange(1, longest + 1)
            rows.append((-1, length, length - 1))
    return rows


@functools.lru_cache(maxsize=8)
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


def _pairs(fresh, cached, window):
    """Visible (query, key) pairs of one request."""
    pos = np.arange(cached, cached + fresh, dtype=np.int64) + 1
    return int(np.minimum(pos, window).sum() if window else pos.sum())


def work(case):
    if case["op"] == "tables":
        rows = _shape_of(case)
        block = case["block"]
        fresh = sum(n - c for _, n, c in rows)
        entries = sum(-(-n // block) - (0 if node >= 0 else -(-c // block)) for node, n, c in rows)
        new = sum(-(-n // block) - -(-c // block) for _, n, c in rows)
        # length, cached, node in, q_start out; table entries; free ids; slot and position a token
        return {"bytes": 16 * len(rows) + 4 * entries + 4 * new + 12 * fresh, "flops": 0}
    row = case["kv_heads"] * case["dim"] * 2
    if case["op"] == "write":
        return {"bytes": case["tokens"] * (4 * row + 8), "flops": 0}
    lens = _lengths(case["requests"], case["fresh"], case["cached"], case["shape"])
    window = case["window"]
    pairs = sum(_pairs(f, c, window) for f, c in lens)
    keys = sum((min(f + c, f + window - 1) if window else f + c) for f, c in lens if f)
    tokens = sum(f for f, _ in lens)
    return {"bytes": 2 * row * keys + 4 * tokens * case["heads"] * case["dim"]
            + 4 * sum(-(-(f + c) // case["block"]) for f, c in lens),
            "flops": 4 * case["dim"] * case["heads"] * pairs}


def _shape_of(case):
    return _table_shape(case["requests"], case["admitted"], case["chunks"], case["depth"], case["block"],
                        case["longest"], case["shape"])


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float16


def _cache(case, blocks, gen):
    """[blocks][block][kv_heads][dim], tokens outside heads or (a view) heads outside tokens."""
    b, h, d = case["block"], case["kv_heads"], case["dim"]
    shape = (blocks, b, h, d) if case["order"] == "token" else (blocks, h, b, d)
    t = torch.empty(shape, dtype=_dtype(case), device="cuda").normal_(generator=gen)
    return t if case["order"] == "token" else t.transpose(1, 2)


def _handle(cache):
    if not own:
        return None
    from paper_2608_01655_gb300 import binding as pp
    return pp.KVCache.like(cache)


def _i32(a):
    return torch.tensor(np.asarray(a, np.int32), device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    rng = np.random.default_rng(seed)
    return {"tables": _prepare_tables, "write": _prepare_write, "attend": _prepare_attend}[case["op"]](case, gen, rng)


def _prepare_tables(case, gen, rng):
    block, requests = case["block"], case["requests"]
    rows = [_shape_of(case)[i] for i in rng.permutation(requests)]
    node, length, cached = (np.array([row[i] for row in rows]) for i in range(3))
    _, unit, used, hops = _tree(case["chunks"], case["depth"], case["shape"])
    per = CHUNK_TOKENS // block
    chunk_map = unit.copy()
    chunk_map[:, 1:] *= per
    chunk_map[unit[:, 1] < 0, 1] = -1
    need, have = -(-length // block), -(-cached // block)
    new = int((need - have).sum())
    width = int(need.max()) + 3
    # blocks: the resident chunks', those of the running requests, and the free ones in any order
    held = int(have[node < 0].sum())
    blocks = used * per + held + new + 17
    other = rng.permutation(np.arange(used * per, blocks))
    table = np.full((requests, width), -1)
    at = 0
    for r in np.flatnonzero(node < 0):
        table[r, :have[r]] = other[at:at + have[r]]
        at += have[r]
    tokens = int((length - cached).sum())
    capacity = -(-tokens // 64) * 64                     # a step's buffers are padded
    cache = torch.empty((blocks, block, 1, 8), dtype=torch.bfloat16, device="cuda") if own else None
    return dict(case=case, block=block, hops=hops, kv=_handle(cache), node=_i32(node), length=_i32(length),
                cached=_i32(np.where(node < 0, cached, 0)), chunk_map=_i32(chunk_map), free=_i32(other[at:]),
                head=_i32([3]), head_out=_i32([0]), table=_i32(table),
                slot=torch.empty(capacity, dtype=torch.int64, device="cuda"),
                position=torch.empty(capacity, dtype=torch.int32, device="cuda"),
                q_start=torch.empty(requests + 1, dtype=torch.int32, device="cuda"))


def _prepare_write(case, gen, rng):
    tokens, h, d = case["tokens"], case["kv_heads"], case["dim"]
    blocks = -(-tokens * 5 // 4 // case["block"]) + 2
    kc, vc = _cache(case, blocks, gen), _cache(case, blocks, gen)
    # K and V are slices of the projection's output beside the queries
    qkv = torch.empty((tokens, 4 * h * d), dtype=_dtype(case), device="cuda").normal_(generator=gen)
    k = qkv[:, 2 * h * d:3 * h * d].unflatten(1, (h, d))
    v = qkv[:, 3 * h * d:].unflatten(1, (h, d))
    # runs of tokens in blocks of any order; some tokens are padding
    order = torch.randperm(blocks, generator=gen, device="cuda")
    slot = (order[:, None] * case["block"] + torch.arange(case["block"], device="cuda")).flatten()
    slot = slot[5:5 + tokens].contiguous()
    slot[torch.arange(tokens, device="cuda") % 37 == 36] = -1
    return dict(case=case, kv=_handle(kc), k=k, v=v, slot=slot, kc=kc, vc=vc)


def _prepare_attend(case, gen, rng):
    lens = _lengths(case["requests"], case["fresh"], case["cached"], case["shape"])
    lens = [lens[i] for i in rng.permutation(len(lens))]
    block, h, d = case["block"], case["kv_heads"], case["dim"]
    fresh = [f for f, _ in lens]
    length = [f + c for f, c in lens]
    need = [-(-n // block) for n in length]
    blocks = sum(need) + 5
    kc, vc = _cache(case, blocks, gen), _cache(case, blocks, gen)
    # keys share a direction and queries are long: softmax weights are spread over decades
    kc += torch.randn((h, d), generator=gen, device="cuda").to(kc.dtype) * 0.5
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
    kc[empty // block, empty % block] = float("nan")
    vc[empty // block, empty % block] = float("nan")
    tokens = sum(fresh)
    # the queries are a slice of the projection's output
    qkv = torch.empty((tokens, (case["heads"] + 2 * h) * d), dtype=_dtype(case), device="cuda")
    qkv = qkv.normal_(generator=gen).mul_(2)
    q = qkv[:, :case["heads"] * d].unflatten(1, (case["heads"], d))
    return dict(case=case, kv=_handle(kc), q=q, kc=kc, vc=vc, table=_i32(table),
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
        return {"tables": _own_tables, "write": _own_write, "attend": _own_attend}[op](pp, state)
    return {"tables": _plain_tables, "write": _plain_write, "attend": _plain_attend}[op](state)


def _own_tables(pp, s):
    pp.pp_block_tables(s["kv"], s["length"], s["cached"], s["table"], s["slot"], s["position"], s["q_start"],
                       s["free"], s["head"], s["head_out"], node=s["node"], chunk_map=s["chunk_map"])
    return {key: s[key] for key in ("table", "slot", "position", "q_start", "head_out")}


def _own_write(pp, s):
    pp.pp_kv_write(s["kv"], s["k"], s["v"], s["slot"], s["kc"], s["vc"])
    return {"kc": s["kc"], "vc": s["vc"]}


def _own_attend(pp, s):
    pp.pp_paged_attention(s["kv"], s["q"], s["kc"], s["vc"], s["table"], s["q_start"], s["length"], s["max_q"],
                          s["out"], s["scale"], window=s["case"]["window"], lse=s["lse"])
    return {"out": s["out"], "lse": s["lse"]}


def _plain_tables(s):
    block, table, length = s["block"], s["table"], s["length"].long()
    width, capacity = table.shape[1], s["slot"].shape[0]
    rec = s["chunk_map"].long()
    node = s["node"].long()
    admitted = node >= 0
    up = torch.where(rec[node.clamp(min=0), 1] >= 0, node, rec[node.clamp(min=0), 0])
    up = torch.where(admitted, up, -1)
    resident = torch.where(up >= 0, rec[up.clamp(min=0), 3], 0) * block
    whole = (length - 1).clamp(min=0) // block * block
    cached = torch.where(admitted, torch.minimum(resident, whole), s["cached"].long())
    fresh = length - cached
    ends = fresh.cumsum(0)
    have, need = (cached + block - 1) // block, (length + block - 1) // block
    new_ends = (need - have).cumsum(0)
    j = torch.arange(width, device=table.device)[None]
    cur = up
    for _ in range(s["hops"]):
        seg = rec[cur.clamp(min=0)][:, :, None]
        hit = (cur >= 0)[:, None] & (j >= seg[:, 2]) & (j < seg[:, 3]) & (j < have[:, None])
        table = torch.where(hit, (seg[:, 1] + j - seg[:, 2]).int(), table)
        cur = torch.where(cur >= 0, seg[:, 0, 0], -1)
    at = s["head"] + (new_ends - (need - have))[:, None] + j - have[:, None]
    new = (j >= have[:, None]) & (j < need[:, None])
    table = torch.where(new, s["free"][at.clamp(0, s["free"].shape[0] - 1)], table)
    t = torch.arange(capacity, device=table.device)
    r = torch.searchsorted(ends, t, right=True).clamp(max=length.shape[0] - 1)
    live = t < ends[-1]
    pos = torch.where(live, cached[r] + t - (ends - fresh)[r], 0)
    slot = torch.where(live, table[r, pos // block].long() * block + pos % block, -1)
    return {"table": table, "slot": slot, "position": pos.int(),
            "q_start": torch.cat([ends.new_zeros(1), ends]).int(), "head_out": (s["head"] + new_ends[-1]).int()}


def _plain_write(s):
    block = s["case"]["block"]
    rows = (s["slot"] >= 0).nonzero()[:, 0]
    slot = s["slot"][rows]
    s["kc"][slot // block, slot % block] = s["k"][rows]
    s["vc"][slot // block, slot % block] = s["v"][rows]
    return {"kc": s["kc"], "vc": s["vc"]}


def _plain_attend(s):
    case = s["case"]
    group, window = case["heads"] // case["kv_heads"], case["window"]
    out, lse = torch.empty_like(s["out"]), torch.empty_like(s["lse"])
    at = 0
    for r, (fresh, n) in enumerate(zip(s["fresh_host"], s["length_host"])):
        if not fresh:
            continue
        ids = s["table"][r, :-(-n // case["block"])].long()
        k = s["kc"][ids].flatten(0, 1)[:n].float().permute(1, 2, 0)             # [h][d][n]
        v = s["vc"][ids].flatten(0, 1)[:n].float().transpose(0, 1)              # [h][n][d]
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
    if case["op"] == "attend":
        return _exact_attend(case, state)
    if case["op"] == "write":
        kc, vc = state["kc"].double(), state["vc"].double()
        slot = state["slot"].cpu().numpy()
        rows = np.flatnonzero(slot >= 0)
        where = (torch.tensor(slot[rows] // case["block"], device="cuda"),
                 torch.tensor(slot[rows] % case["block"], device="cuda"))
        rows = torch.tensor(rows, device="cuda")
        return {"kc": kc.index_put(where, state["k"].double()[rows]),
                "vc": vc.index_put(where, state["v"].double()[rows])}
    return _exact_tables(case, state)


def _exact_tables(case, state):
    """One request after another, on the host."""
    block = case["block"]
    host = {k: v.cpu().numpy().astype(np.int64) for k, v in state.items() if torch.is_tensor(v)}
    table, rec, head = host["table"], host["chunk_map"], int(host["head"][0])
    slot, position = np.full(len(host["slot"]), -1), np.zeros(len(host["slot"]), np.int64)
    q_start = [0]
    for r, (node, n, cached) in enumerate(zip(host["node"], host["length"], host["cached"])):
        n = int(n)
        if node >= 0:
            chunk = node if rec[node, 1] >= 0 else rec[node, 0]
            cached = min(rec[chunk, 3] * block if chunk >= 0 else 0, max(n - 1, 0) // block * block)
            while chunk >= 0:
                up, base, begin, end = rec[chunk]
                end = min(end, cached // block)
                if end > begin:
                    table[r, begin:end] = base + np.arange(end - begin)
                chunk = up
        cached = int(cached)
        for j in range(-(-cached // block), -(-n // block)):
            table[r, j] = host["free"][head]
            head += 1
        pos = np.arange(cached, n)
        at = slice(q_start[-1], q_start[-1] + n - cached)
        position[at] = pos
        slot[at] = table[r, pos // block] * block + pos % block
        q_start.append(at.stop)
    as_tensor = lambda a: torch.tensor(np.asarray(a, np.int64), device="cuda")
    return {"table": as_tensor(table), "slot": as_tensor(slot), "position": as_tensor(position),
            "q_start": as_tensor(q_start), "head_out": as_tensor([head])}


def _exact_attend(case, state):
    block, group, window = case["block"], case["heads"] // case["kv_heads"], case["window"]
    out = torch.empty(state["out"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(state["lse"].shape, dtype=torch.float64, device="cuda")
    start = 0
    for r, (fresh, n) in enumerate(zip(state["fresh_host"], state["length_host"])):
        j = torch.arange(n, device="cuda")
        page = state["table"][r].long()[j // block]
        for h in range(case["kv_heads"]):
            k = state["kc"][page, j % block, h].double()
            v = state["vc"][page, j % block, h].double()
            for a in range(0, fresh, 1024):
                b = min(fresh, a + 1024)
                p = torch.arange(n - fresh + a, n - fresh + b, device="cuda")[:, None]
                seen = j[None] <= p
                if window:
                    seen &= j[None] > p - window
                for g in range(h * group, (h + 1) * group):
                    rows = slice(start + a, start + b)
                    s = (state["q"][rows, g].double() @ k.T) * state["scale"]
                    s = torch.where(seen, s, -math.inf)
                    lse[rows, g] = torch.logsumexp(s, 1)
                    out[rows, g] = torch.exp(s - lse[rows, g][:, None]) @ v
        start += fresh
    return {"out": out, "lse": lse}
