"""Few rows over an 8-bit cache whose weights lie many powers of two apart: what many small ones
add up to is part of the output, whatever the scales of the blocks beside them."""
import math

import numpy as np
import pytest

from tests import kv8_reference as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

BF, HF = torch.bfloat16, torch.float16

# A weight is at most 2^15 as an operand, so that f16's half step at the bottom, 2^-25, is 2^-40
# of the largest; 11 bits stay down to 2^-29 of it.
LOST = 2.0 ** -40


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


def _run(pp, requests, length, heads, kv_heads, dim, dtype, tail, gap, strong, seed=0):
    """Blocks of 16 keys.  In the first `strong` of them, which all requests share, the first key scores `tail`
    powers of two (of its weight) above all other keys, and V's element 0 of that key is 448 * 2^gap, which sets its
    block's scale; its other elements are 0.  V is near 1 in all other keys."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    need = -(-length // 16)
    blocks = 2 * need + 1
    kc = torch.zeros((blocks, 16, kv_heads, dim), device="cuda")
    vc = 1 + 0.5 * torch.rand((blocks, 16, kv_heads, dim), generator=gen, device="cuda")
    kc[:strong, 0, :, 0] = 1.0
    vc[:strong, 0] = 0.0
    vc[:strong, 0, :, 0] = 448 * 2.0 ** gap
    (kc, ke), (vc, ve) = ref.to8(kc), ref.to8(vc)
    q = torch.zeros((requests, heads, dim), dtype=dtype, device="cuda")
    q[:, :, 0] = tail                                       # a score of tail * ln 2
    scale = math.log(2.0)
    table = np.tile(np.arange(need), (requests, 1))
    table[1::2, strong:] += need
    out = torch.empty_like(q)
    lse = torch.empty((requests, heads), device="cuda")
    q_start, lengths = list(range(requests + 1)), [length - r % 5 for r in range(requests)]
    with pp.KVCache.like(kc, dtype=dtype) as kv:
        pp.pp_paged_attention8(kv, q, kc, ke, vc, ve, _i32(table), _i32(q_start), _i32(lengths), 1, out, scale, lse=lse)
        kv.sync()
    some = [0, 1, 2, requests - 1]
    want, wl, tol, ltol = ref.attention8(q[some], kc, ke, vc, ve, _i32(table[some]), list(range(5)), [lengths[r] for r in some],
                                         scale, 0, True, LOST)
    got = out[some].double()
    err, lerr = (got - want).abs(), (lse[some].double() - wl).abs()
    if dtype == HF:                                         # numbers from 65520 on round to f16's infinity
        far = want - tol >= 65520
        assert (got[far] == math.inf).all()
        err[far] = 0
    assert (err <= tol).all(), f"worst {float((err / tol).max())} of its bound, {float((err / want.abs().clamp(min=1e-30)).max())} of its value"
    assert (lerr <= ltol).all()
    return want, tol


@pytest.mark.parametrize("heads,dim,dtype", [(8, 128, BF), (1, 64, HF), (16, 64, BF), (40, 128, HF)])
@pytest.mark.parametrize("tail,gap", [(17, 8), (12, 14), (25, 0), (3, 20)])
def test_a_tail_beside_strong_keys_in_blocks_of_large_scale(pp, heads, dim, dtype, tail, gap):
    """Requests that a CTA has whole, with a strong key in the first tile of every warp.  (The first 24 blocks; a tile
    has 12 or 8.)"""
    want, tol = _run(pp, 320, 4001, heads, 1, dim, dtype, tail, gap, 24)
    assert (want[..., 1:] > 8 * tol[..., 1:]).all()         # a lost tail would be seen


@pytest.mark.parametrize("tail,gap", [(17, 8), (25, 0)])
def test_a_long_tail_in_pieces(pp, tail, gap):
    _run(pp, 4, 150_001, 8, 2, 128, BF, tail, gap, 9000)


@pytest.mark.parametrize("gap", [-30, 30])
def test_scales_that_push_weights_to_the_ends(pp, gap):
    """The strong keys' values 2^30 below and above the others': weights of either kind fall off the other's."""
    _run(pp, 200, 701, 8, 2, 64, BF, 10, gap, 30)


@pytest.mark.parametrize("size", [10, 20, 22, 23, 24, 25, 26, 27, 28, 30, 34, 50])
@pytest.mark.parametrize("heads", [1, 9])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_scores_of_any_size(pp, size, heads, dtype):
    """One key far above the others, at 2^size and more: its V row is the output however coarse the scores' steps are.
    Keys come in an order in which the maximum moves many times, by small and large steps."""
    gen = torch.Generator(device="cuda").manual_seed(size)
    blocks, dim = 90, 64
    kc, vc = (torch.rand((blocks, 16, 1, dim), generator=gen, device="cuda") for _ in range(2))
    kc[..., 0] = torch.linspace(0.25, 0.5, blocks * 16, device="cuda").view(blocks, 16, 1)
    kc[77, 5, 0, 0] = 1.0
    (kc, ke), (vc, ve) = ref.to8(kc), ref.to8(vc)
    assert (ke == -8).all()
    ke += torch.tensor(size - 20 + 8, dtype=torch.int8, device="cuda").clamp(max=48)
    rest = 2.0 ** (size - int(ke[0, 0]) - 8)                # what the exponents leave to the scale
    q = torch.zeros((2, heads, dim), dtype=dtype, device="cuda")
    q[..., 0] = torch.arange(1, heads + 1, device="cuda")
    out, lse = torch.empty_like(q), torch.empty((2, heads), device="cuda")
    table, length = [list(range(blocks))] * 2, [blocks * 16, blocks * 16 - 77]
    with pp.KVCache.like(kc, dtype=dtype) as kv:
        pp.pp_paged_attention8(kv, q, kc, ke, vc, ve, _i32(table), _i32([0, 1, 2]), _i32(length), 1, out, rest, lse=lse)
        kv.sync()
    v = ref.scaled(vc, ve)[77, 5, 0]
    u = ref.UNIT[dtype]
    # the next key is 2^(size - 2) behind; weights and sums of one key cancel but for roundings of 2^-11 and 2^-20
    assert ((out.double() - v).abs() <= 1.01 * (u + 2.0 ** -11 + 2.0 ** -20) * v.abs() + ref.TINY[dtype]).all()
    score = q[..., 0].double() * ref.scaled(kc, ke)[77, 5, 0, 0] * rest
    assert float(score.min()) >= 2.0 ** size * 0.99
    assert ((lse.double() - score).abs() <= score * 2.0 ** -20).all()
