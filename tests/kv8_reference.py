"""Plain 64-bit forms of the rotation, the 8-bit cache's write and attention over it, and
error bounds that follow from the types and sizes alone."""
import math

import numpy as np
import torch

LEAST, MOST = -40, 40
UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}


# ---------------------------------------------------------------------------
# Rotation
# ---------------------------------------------------------------------------
def rotate(x, weight, eps, position, frequencies, rotated, interleaved, amplitude):
    """Rows [T][heads][dim] in 64 bits and bounds of their errors.

    In 32 bits: a norm's sum of dim squares is off by dim 2^-24 of itself, so its root by
    half of that; 2^-20 covers the root, the divisions and products (8 roundings).  An
    angle is off by 2^-23 rad (a fraction of a turn rounded to 24 bits), cos and sin by
    2^-23 more, and products and their sum by 3 roundings: 2^-21 of |y_a| + |y_b|.  Then
    one rounding to the type."""
    t, heads, dim = x.shape
    y = x.double()
    off = torch.zeros_like(y)
    if weight is not None:
        y = y / torch.sqrt(y.square().mean(-1, keepdim=True) + eps) * weight.double()
        off = y.abs() * (dim * 2.0 ** -25 + 2.0 ** -20)
    half = rotated // 2
    i = torch.arange(half, device=x.device)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    angle = position.double()[:, None, None] * torch.as_tensor(np.asarray(frequencies), device=x.device).double()
    cos, sin = torch.cos(angle) * amplitude, torch.sin(angle) * amplitude
    out, tol = y.clone(), off.clone()
    out[..., a] = y[..., a] * cos - y[..., b] * sin
    out[..., b] = y[..., b] * cos + y[..., a] * sin
    size = abs(amplitude) * 2.0 ** -21 * (y[..., a].abs() + y[..., b].abs()) + abs(amplitude) * (off[..., a] + off[..., b])
    tol[..., a], tol[..., b] = size, size
    tol = 1.01 * (tol + UNIT[x.dtype] * (out.abs() + tol) + TINY[x.dtype])
    if weight is None:
        tol[..., rotated:] = 0                              # bits are kept
    return out, tol


# ---------------------------------------------------------------------------
# The cache
# ---------------------------------------------------------------------------
def e4m3(y):
    """The nearest e4m3 numbers, ties to even, saturated; NaN stays."""
    y = np.asarray(y, np.float64)
    size = np.abs(np.where(np.isfinite(y) & (y != 0), y, 1.0))
    step = np.exp2(np.maximum(np.floor(np.log2(size)), -6) - 3)
    return np.clip(np.round(y / step) * step, -448, 448)


def values(code):
    """float8_e4m3fn numbers of any shape as 64-bit ones, on the host."""
    return code.view(torch.uint8).cpu().clone().view(torch.float8_e4m3fn).double().numpy()


def write8(x, slot, code, exponent, block):
    """One of K and V: rows x [T][heads][dim] (64-bit, host) into code [blocks][block][heads][dim] (values) and
    exponent [blocks][heads]; new ones are returned."""
    code, exponent = code.copy(), exponent.astype(np.int64)
    rows = {}
    for t, s in enumerate(slot):
        if 0 <= s < code.shape[0] * block:
            rows.setdefault(int(s) // block, []).append((int(s) % block, t))
    for b, some in rows.items():
        places = [p for p, _ in some]
        others = [p for p in range(block) if p not in places]
        for h in range(x.shape[1]):
            new = np.stack([x[t, h] for _, t in some])
            finite = np.abs(new[np.isfinite(new)])
            top = finite.max() if finite.size else 0.0
            need = LEAST
            while need < MOST and top > 448 * 2.0 ** need:
                need += 1
            old = min(max(int(exponent[b, h]), LEAST), MOST)
            e = need if 0 in places else max(old, need)
            if 0 not in places and e > old:
                code[b, others, h] = e4m3(code[b, others, h] * 2.0 ** (old - e))
            code[b, places, h] = e4m3(np.where(np.isfinite(new), new, np.nan) * 2.0 ** -e)
            exponent[b, h] = e
    return code, exponent


def scaled(code, exponent):
    """Codes times 2^exponent, 64-bit, on the device of `code`."""
    e = exponent.double().clamp(LEAST, MOST)
    return code.view(torch.uint8).contiguous().view(torch.float8_e4m3fn).double() * torch.exp2(e)[:, None, :, None]


# ---------------------------------------------------------------------------
# Attention
# ---------------------------------------------------------------------------
def attention8(q, kc, ke, vc, ve, table, q_start, length, scale, window, direct, lost=2.0 ** -25):
    """out and lse in 64 bits, and bounds of their errors.  direct: the kernel that reads codes; else that of
    rows unpacked to q's type.  lost: the largest error of a weight below its 16-bit type's normal range, of the
    largest w_j 2^ve_j (direct).

    With u the unit roundoff of the type, D the head dimension, w_j the weights
    relative to the largest and l = sum w_j >= 1:
      scores   |ds| <= scale D 2^-23 max_j sum |q k| for sums in 32 bits and scaling;
               direct: bf16 queries lose 2^-38 of the row's largest element, and the
               exponent beside a score rounds |s| + 40 by 2^-24, 2^-18 for both with
               the exponential; unpacked f16: 2^-25 of each k;
               a weight's relative error is 2 c at most;
      weights  direct: 2^-11 w |v| each, and below f16's normal range, whose unit is the
               largest w_j 2^ve_j, `lost` of that times the code;
               unpacked: u w |v|, in f16 below its normal range 2^-25 |v|;
      V        unpacked f16: 2^-25;
      output   u |o|, in f16 at least 2^-25."""
    dtype, dev = q.dtype, q.device
    u, tiny = UNIT[dtype], TINY[dtype]
    tokens, heads, dim = q.shape
    block, kv_heads = kc.shape[1], kc.shape[2]
    group = heads // kv_heads
    out = torch.zeros((tokens, heads, dim), dtype=torch.float64, device=dev)
    lse = torch.full((tokens, heads), -math.inf, dtype=torch.float64, device=dev)
    out_tol, lse_tol = torch.zeros_like(out), torch.zeros_like(lse)
    for r in range(len(length)):
        a, b, n = int(q_start[r]), int(q_start[r + 1]), int(length[r])
        if a == b or n <= 0:
            continue
        j = torch.arange(n, device=dev)
        pages, inv = torch.unique(table[r].long()[j // block], return_inverse=True)
        size = torch.exp2(ve[pages].double().clamp(LEAST, MOST))                          # [pages][h]
        k, v = (scaled(c.view(torch.uint8)[pages].view(torch.float8_e4m3fn), e[pages]) for c, e in ((kc, ke), (vc, ve)))
        k = k[inv, j % block].permute(1, 2, 0)                                            # [h][d][n]
        v = v[inv, j % block].transpose(0, 1)                                             # [h][n][d]
        size = size[inv].transpose(0, 1)                                                  # [h][n]
        for x in range(a, b):
            p = n - (b - a) + (x - a)
            lo = max(0, p - window + 1) if window else 0
            if p < 0:
                continue
            kk, vv, sz = k[:, :, lo:p + 1], v[:, lo:p + 1], size[:, None, lo:p + 1]
            qq = q[x].double().view(kv_heads, group, dim)
            s = torch.matmul(qq, kk) * scale
            c = scale * dim * 2.0 ** -23 * torch.matmul(qq.abs(), kk.abs()).amax(-1)      # [h][g]
            mass_k = kk.abs().sum(1).amax(-1)[:, None]
            if direct:
                c = c + scale * 2.0 ** -38 * qq.abs().amax(-1) * mass_k + 2.0 ** -18
            else:
                c = c + tiny * scale * qq.abs().sum(-1)
            top = s.amax(-1, keepdim=True)
            w = torch.exp(s - top)
            l = w.sum(-1, keepdim=True)
            o = torch.matmul(w, vv) / l
            mass = torch.matmul(w, vv.abs()) / l
            out[x] = o.reshape(heads, dim)
            lse[x] = (top + l.log()).reshape(heads)
            lse_tol[x] = c.reshape(heads) + 2.0 ** -20 * (1 + lse[x].abs())
            if direct:
                unit = (w * sz).amax(-1, keepdim=True)                                    # what a weight of 1 stands for
                low = lost * unit * (vv.abs() / sz.transpose(1, 2)).sum(1)[:, None] / l
                weights = 2.0 ** -11 * mass + low
            else:
                weights = u * mass + tiny * (vv.abs().sum(1)[:, None] / l + 1)
            tol = u * o.abs() + tiny + weights + (2 * c[..., None] + 2.0 ** -20) * mass
            out_tol[x] = 1.01 * tol.reshape(heads, dim)
    return out, lse, out_tol, lse_tol


def to8(x):
    """A cache of any numbers [blocks][block][heads][dim] as codes and exponents, on its device."""
    top = x.double().abs().amax((1, 3))
    fraction, power = torch.frexp(top)
    e = (power - 9 + (fraction > 0.875)).clamp(LEAST, MOST)
    code = (x.double() * torch.exp2(-e.double())[:, None, :, None]).float().clamp(-448, 448).to(torch.float8_e4m3fn)
    return code, e.to(torch.int8)
