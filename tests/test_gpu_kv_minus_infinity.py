"""Scores of -infinity: a query all of whose visible keys have that score has 0 / 0 in every
column by the definition and the log of an empty sum; one that sees a finite score has its
weights there; one that sees no key has zeros."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def pp():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_01655_gb300 import build
    build.build()
    from paper_2608_01655_gb300 import binding
    return binding


def _i32(a):
    return torch.tensor(np.asarray(a, np.int32), device="cuda")


@pytest.mark.parametrize("dim,dtype", [(64, torch.float16), (128, torch.bfloat16), (40, torch.bfloat16)])
@pytest.mark.parametrize("fresh,length", [([1, 1], [300, 40]), ([3, 2], [9000, 2]), ([200, 70], [700, 20]),
                                          ([40, 1], [20_000, 1]), ([2], [4]), ([130], [100])])
@pytest.mark.parametrize("finite", [False, True])
def test_scores_of_minus_infinity(pp, dim, dtype, fresh, length, finite):
    torch.manual_seed(13)
    heads, kv_heads = 4, 2
    need = [-(-n // 16) for n in length]
    kc, vc = (torch.randn((sum(need), 16, kv_heads, dim), device="cuda").to(dtype) for _ in range(2))
    kc[..., 0] = math.inf
    table, at = np.zeros((len(fresh), max(need))), 0
    for r, n in enumerate(need):
        table[r, :n] = np.arange(at, at + n)
        if finite:
            kc[at, 0, :, 0] = 1                             # each request's first key
        at += n
    q = torch.randn((sum(fresh), heads, dim), device="cuda").to(dtype)
    q[..., 0] = -1
    out, lse = torch.full_like(q, 7), torch.full(q.shape[:2], 7.0, device="cuda")
    with pp.KVCache.like(kc) as kv:
        pp.pp_paged_attention(kv, q, kc, vc, _i32(table), _i32(np.concatenate([[0], np.cumsum(fresh)])), _i32(length),
                              max(fresh), out, 0.125, lse=lse)
        kv.sync()
    first, row = 0, 0
    for r, (f, n) in enumerate(zip(fresh, length)):
        blind = max(0, f - n)                               # queries before the first key
        assert (out[row:row + blind] == 0).all() and (lse[row:row + blind] == -math.inf).all()
        some = slice(row + blind, row + f)
        if finite:
            v = vc[first, 0].repeat_interleave(heads // kv_heads, 0)
            assert torch.equal(out[some], v.expand(out[some].shape)) and lse[some].isfinite().all()
        else:
            assert out[some].isnan().all() and (lse[some] == -math.inf).all()
        first += need[r]
        row += f
