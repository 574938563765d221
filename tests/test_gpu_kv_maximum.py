"""The running maximum of the softmax, at sizes where every CTA has several tiles of an item:
scores whose level changes from tile to tile, so that sums and outputs are rescaled between
them, and scores that are all -infinity.  Against the 64-bit form within its bound."""
import math

import numpy as np
import pytest

from tests import kv_reference as ref
from tests.kv_tiles import chunk_tiles, token_tiles

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


def _within(got, want, tol):
    """Also false where `got` is NaN."""
    return bool(((got.double() - want).abs() <= tol).all())


# log2 of the weights' level in tile t of the keys
LEVELS = {
    "steps": lambda t: 1.2 * t,                 # several tiles between two moves: what is rescaled still counts
    "climb": lambda t: 14.0 * t,                # each tile outweighs all before it by more than 2^12
    "fall": lambda t: -3.0 * t,                 # the first maximum stands
    "saw": lambda t: 1.1 * t + (t % 3 == 2) * 9.0,
    "jump": lambda t: 0.4 * t + (t >= 11) * 60.0,
}


def _cache(levels, kv_heads, dim, dtype):
    n = len(levels)
    k = torch.randn((n, kv_heads, dim), device="cuda") * 0.4
    k += torch.tensor(levels, device="cuda", dtype=torch.float32)[:, None, None] / dim
    v = torch.randn((n, kv_heads, dim), device="cuda") + torch.randn((kv_heads, dim), device="cuda")
    return [x.to(dtype).unflatten(0, (-1, 16)) for x in (k, v)]


@pytest.mark.parametrize("level", LEVELS)
@pytest.mark.parametrize("fresh,cached,kv_heads,heads", [([1000, 300], [2000, 2900], 8, 16), ([1] * 6, [4000] * 6, 8, 16),
                                                         ([2, 3, 1, 3, 2, 3], [4000] * 6, 8, 16)])
@pytest.mark.parametrize("dim,dtype", [(128, torch.bfloat16), (64, torch.float16), (64, torch.bfloat16), (80, torch.float16)])
def test_levels_that_change_between_tiles(pp, level, fresh, cached, kv_heads, heads, dim, dtype):
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    count = token_tiles if max(fresh) * (heads // kv_heads) <= 32 else chunk_tiles
    assert count(fresh, cached, heads // kv_heads, kv_heads) >= 8 * sms
    torch.manual_seed(12)
    length = [f + c for f, c in zip(fresh, cached)]
    n = -(-max(length) // 128) * 128
    kc, vc = _cache([LEVELS[level](j // 128) for j in range(n)], kv_heads, dim, dtype)
    # all requests over the same blocks, each with rows of its own
    table = torch.arange(n // 16, dtype=torch.int32, device="cuda").repeat(len(fresh), 1)
    q = (1 + 0.2 * torch.randn((sum(fresh), heads, dim), device="cuda")).to(dtype)
    q_start = np.concatenate([[0], np.cumsum(fresh)])
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    with pp.KVCache.like(kc) as kv:
        pp.pp_paged_attention(kv, q, kc, vc, table, _i32(q_start), _i32(length), max(fresh), out, math.log(2.0), lse=lse)
        kv.sync()
    want, want_lse, tol, lse_tol = ref.attention(q, kc, vc, table, q_start, length, math.log(2.0), 0)
    assert _within(out, want, tol) and _within(lse, want_lse, lse_tol)
