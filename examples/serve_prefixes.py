"""Serve from a planned target: from pp_plan_run to attention over the worker's cache.

    python examples/serve_prefixes.py [requests [decode steps]]

Plans the tiny workload, lays worker 0's resident chunks out as blocks of a paged
K/V cache (pp_chunk_map) and stores their rows.  Then requests arrive whose
prompts end in chunks of the tree, with tails of their own: one step admits them
(pp_block_tables takes what is resident from the cache, pp_kv_write stores the
rest's rows, pp_paged_attention attends the rest), and the steps after it add a
token to each.  The model is one attention layer with random weights over
embeddings of token and position; what the cached rows give is compared with
attention over whole prompts computed anew.
"""
import math
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2608_01655_gb300 import binding as pp    # noqa: E402
from paper_2608_01655_gb300 import workloads as wl  # noqa: E402

SLOT_TOKENS, BLOCK = 512, 16
HEADS, KV_HEADS, DIM, HIDDEN, VOCABULARY = 16, 2, 128, 256, 4096


class Layer:
    """q, k and v of tokens at positions."""

    def __init__(self):
        gen = torch.Generator(device="cuda").manual_seed(1)
        rand = lambda *shape: torch.randn(shape, generator=gen, device="cuda")
        self.embedding, self.place = rand(VOCABULARY, HIDDEN), rand(64, HIDDEN)
        self.weight = rand(HIDDEN, (HEADS + 2 * KV_HEADS) * DIM).mul_(1.5 / HIDDEN ** 0.5)

    def __call__(self, token, position):
        x = self.embedding[token] + self.place[position % 64]
        qkv = (x @ self.weight).to(torch.bfloat16).unflatten(1, (-1, DIM))
        return qkv.split((HEADS, KV_HEADS, KV_HEADS), dim=1)


def chunk_tokens(chunk, count):
    return (chunk * 40_503 + np.arange(count) * 977) % VOCABULARY


def path_of(parent, chunk):
    path = []
    while chunk >= 0:
        path.append(chunk)
        chunk = int(parent[chunk])
    return path[::-1]


def run(requests=24, steps=4, seed=0):
    torch.cuda.set_device(0)
    rng = np.random.default_rng(seed)
    inst = wl.make(0)
    with pp.Instance.from_workload(inst) as ppi:
        plan = pp.pp_plan_run(ppi, inst.starts, None, inst.rounds)
    resident = plan.placement[0]
    per_slot = SLOT_TOKENS // BLOCK
    chunk_map, used = pp.pp_chunk_map(inst.parent, inst.weight, resident, per_slot)

    # prompts: a path of the tree that the worker is asked for, and a tail
    asked = np.flatnonzero(inst.demand[0] > 0)
    node = rng.choice(asked, size=requests, p=inst.demand[0, asked] / inst.demand[0, asked].sum()).astype(np.int32)
    prompt = []
    for b in node:
        ids = [chunk_tokens(c, SLOT_TOKENS * int(inst.weight[c])) for c in path_of(inst.parent, int(b))]
        prompt.append(np.concatenate(ids + [rng.integers(0, VOCABULARY, size=int(rng.integers(1, 300)))]))
    length = np.array([len(p) for p in prompt], np.int32)
    width = int(-(-(length.max() + steps) // BLOCK))
    sequence = np.zeros((requests, width * BLOCK), np.int64)
    for r, ids in enumerate(prompt):
        sequence[r, :len(ids)] = ids
        sequence[r, len(ids):] = rng.integers(0, VOCABULARY, size=width * BLOCK - len(ids))     # what it will generate
    sequence = torch.tensor(sequence, device="cuda")

    layer = Layer()
    blocks = used + requests * width
    k_cache, v_cache = (torch.empty((blocks, BLOCK, KV_HEADS, DIM), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    i32 = lambda a: torch.tensor(np.asarray(a, np.int32), device="cuda")
    with pp.KVCache.like(k_cache) as kv:
        # the resident chunks' rows, as their materialisation would leave them
        for b in np.flatnonzero(resident):
            count = SLOT_TOKENS * int(inst.weight[b])
            _, base, begin, end = (int(x) for x in chunk_map[b])
            first = end * BLOCK - count
            position = torch.arange(first, first + count, device="cuda")
            _, k, v = layer(torch.tensor(chunk_tokens(b, count), device="cuda"), position)
            pp.pp_kv_write(kv, k, v, position + (base - begin) * BLOCK, k_cache, v_cache)

        table = torch.full((requests, width), -1, dtype=torch.int32, device="cuda")
        free = torch.arange(used, blocks, dtype=torch.int32, device="cuda")
        head, head_out = i32([0]), i32([0])
        q_start = i32(np.zeros(requests + 1))
        tree, nodes = i32(chunk_map), i32(node)
        cached_tokens, worst = 0, 0.0
        for step in range(steps + 1):
            now = length + step
            cached = i32(now - 1)
            capacity = int(now.sum()) if step == 0 else requests
            slot = torch.empty(capacity, dtype=torch.int64, device="cuda")
            position = torch.empty(capacity, dtype=torch.int32, device="cuda")
            admitted = dict(node=nodes, chunk_map=tree) if step == 0 else {}
            now_dev = i32(now)
            pp.pp_block_tables(kv, now_dev, cached, table, slot, position, q_start, free, head, head_out, **admitted)
            head, head_out = head_out, head
            # the host needs the count of new tokens to size what the layer computes
            starts = q_start.cpu().numpy()
            fresh = int(starts[-1])
            request = torch.repeat_interleave(torch.arange(requests, device="cuda"),
                                              (q_start[1:] - q_start[:-1]).long())
            place = position[:fresh].long()
            q, k, v = layer(sequence[request, place], place)
            pp.pp_kv_write(kv, k, v, slot[:fresh], k_cache, v_cache)
            out = torch.empty((fresh, HEADS, DIM), dtype=torch.bfloat16, device="cuda")
            pp.pp_paged_attention(kv, q, k_cache, v_cache, table, q_start, now_dev, int(np.diff(starts).max()), out,
                                  DIM ** -0.5)
            kv.sync()
            if step == 0:
                cached_tokens = int(now.sum()) - fresh
            worst = max(worst, check(layer, sequence, now, starts, out, rng.integers(0, requests, size=4)))
    return dict(requests=requests, resident_chunks=int(resident.sum()), prompt_tokens=int(length.sum()),
                cached_tokens=cached_tokens, blocks=blocks, worst_error=worst)


def check(layer, sequence, length, starts, out, some):
    """The largest difference from attention over the whole prompt in 64 bits, relative to the largest value."""
    worst = 0.0
    for r in some:
        n, a, b = int(length[r]), int(starts[r]), int(starts[r + 1])
        position = torch.arange(n, device="cuda")
        q, k, v = (x.double().transpose(0, 1) for x in layer(sequence[r, :n], position))
        k, v = (x.repeat_interleave(HEADS // KV_HEADS, 0) for x in (k, v))
        score = (q[:, n - (b - a):] @ k.transpose(1, 2)) * DIM ** -0.5
        score.masked_fill_(position > position[n - (b - a):, None], float("-inf"))
        want = (score.softmax(-1) @ v).transpose(0, 1)
        error = float((out[a:b].double() - want).abs().max() / want.abs().max())
        if not math.isfinite(error):                        # max() below would pass over a NaN
            raise ArithmeticError(f"attention gave infinities or NaN for request {r}")
        worst = max(worst, error)
    return worst


if __name__ == "__main__":
    result = run(*(int(x) for x in sys.argv[1:3]))
    print(f"{result['resident_chunks']} chunks resident; of {result['prompt_tokens']} prompt tokens of "
          f"{result['requests']} requests {result['cached_tokens']} came from the cache; largest difference from "
          f"attention over whole prompts {result['worst_error']:.1e}")
