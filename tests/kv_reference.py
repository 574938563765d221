"""Plain 64-bit forms of the paged-cache operators, one request after another,
and error bounds that follow from the types and sizes alone."""
import math

import numpy as np
import torch


def block_tables(length, cached, node, chunk_path_blocks, table, free, head, block, capacity):
    """chunk_path_blocks(node): block ids of the resident chunks on the path of
    `node`, from the root.  Returns (table, slot, position, q_start, head)."""
    table = np.array(table, np.int64)
    slot, position, q_start = [], [], [0]
    for r, n in enumerate(length):
        n, c = int(n), int(cached[r])
        if node is not None and node[r] >= 0:
            shared = chunk_path_blocks(int(node[r]))
            c = min(len(shared) * block, max(n - 1, 0) // block * block)
            table[r, :c // block] = shared[:c // block]
        for j in range(-(-c // block), -(-n // block)):
            table[r, j] = free[head]
            head += 1
        for p in range(c, n):
            slot.append(table[r, p // block] * block + p % block)
            position.append(p)
        q_start.append(len(slot))
    pad = capacity - len(slot)
    return table, np.array(slot + [-1] * pad, np.int64), np.array(position + [0] * pad), np.array(q_start), head


def attention(q, k_cache, v_cache, table, q_start, length, scale, window):
    """out and lse in 64 bits, and bounds of their errors for a kernel that sums
    products in 32 bits, rounds the softmax weights to the cache's type for
    their product with V, and rounds the result once.

    With u the unit roundoff of the type, D the head dimension, w_j the
    weights relative to the largest and l = sum w_j >= 1:
      scores   |ds| <= c = scale D 2^-23 max_j sum |q k|, so a weight's relative
               error is 2 c at most (2^-20 more for exp and the running sums);
      weights  u |v| w each, and in f16 below its normal range 2^-25 |v| each;
      output   u |o|, in f16 at least 2^-25.
    """
    dtype, dev = q.dtype, q.device
    u = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -11
    small = 0.0 if dtype == torch.bfloat16 else 2.0 ** -25
    tokens, heads, dim = q.shape
    block, kv_heads = k_cache.shape[1], k_cache.shape[2]
    group = heads // kv_heads
    out = torch.zeros((tokens, heads, dim), dtype=torch.float64, device=dev)
    lse = torch.full((tokens, heads), -math.inf, dtype=torch.float64, device=dev)
    out_tol, lse_tol = torch.zeros_like(out), torch.zeros_like(lse)
    for r in range(len(length)):
        a, b, n = int(q_start[r]), int(q_start[r + 1]), int(length[r])
        if a == b or n == 0:
            continue
        j = torch.arange(n, device=dev)
        page = table[r].long()[j // block]
        k = k_cache[page, j % block].double().permute(1, 2, 0)        # [h][d][n]
        v = v_cache[page, j % block].double().transpose(0, 1)         # [h][n][d]
        for x in range(a, b):
            p = n - (b - a) + (x - a)
            lo = max(0, p - window + 1) if window else 0
            if p < 0:
                continue
            kk, vv = k[:, :, lo:p + 1], v[:, lo:p + 1]
            qq = q[x].double().view(kv_heads, group, dim)
            s = torch.matmul(qq, kk) * scale
            c = scale * dim * 2.0 ** -23 * torch.matmul(qq.abs(), kk.abs()).amax(-1)     # [h][g]
            top = s.amax(-1, keepdim=True)
            w = torch.exp(s - top)
            l = w.sum(-1, keepdim=True)
            o = torch.matmul(w, vv) / l
            mass = torch.matmul(w, vv.abs()) / l
            out[x] = o.reshape(heads, dim)
            lse[x] = (top + l.log()).reshape(heads)
            lse_tol[x] = c.reshape(heads) + 2.0 ** -20 * (1 + lse[x].abs())
            tol = u * o.abs() + (u + 2 * c[..., None] + 2.0 ** -20) * mass + small * (1 + vv.abs().sum(1)[:, None] / l)
            out_tol[x] = 1.01 * tol.reshape(heads, dim)
    return out, lse, out_tol, lse_tol
