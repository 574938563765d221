"""pp_paged_attention8 where requests share blocks, as those with one prefix do, and with groups of query
heads at the end of what the kernel of single tokens takes; the write's border of a scale."""
import numpy as np
import pytest

from tests import kv8_reference as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

BF, HF = torch.bfloat16, torch.float16


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


def _compare(pp, table, fresh, length, heads, kv_heads, dim, dtype, block, window=0, room=None):
    """Runs the call over the blocks of `table` and compares it with the 64-bit form; returns the output."""
    torch.manual_seed(len(fresh))
    table = np.asarray(table)
    blocks = int(table.max()) + 1
    (kc, ke), (vc, ve) = (ref.to8(torch.randn((blocks, block, kv_heads, dim), device="cuda")
                                  * torch.exp2(torch.randn((blocks, 1, kv_heads, 1), device="cuda"))) for _ in range(2))
    q = (2 * torch.randn((sum(fresh), heads, dim), device="cuda")).to(dtype)
    out, lse = torch.empty_like(q), torch.empty((len(q), heads), device="cuda")
    q_start = np.concatenate([[0], np.cumsum(fresh)])
    seen = sum(-(-n // block) for n in length) if room is None else room
    direct = max(fresh) * (heads // kv_heads) <= 48
    with pp.KVCache.like(kc, dtype=dtype) as kv:
        w = None if direct else torch.empty(kv.workspace_size(len(fresh), table.shape[1], seen), dtype=torch.uint8, device="cuda")
        pp.pp_paged_attention8(kv, q, kc, ke, vc, ve, _i32(table), _i32(q_start), _i32(length), max(fresh), out, dim ** -0.5,
                               window=window, lse=lse, workspace=w)
        kv.sync()
    want, wl, tol, ltol = ref.attention8(q, kc, ke, vc, ve, _i32(table), q_start, length, dim ** -0.5, window, direct)
    err = (out.double() - want).abs()
    assert (err <= tol).all(), f"worst {float((err / tol).max())} of its bound"
    assert ((lse.double() - wl).abs() <= ltol).all()
    return out


def _shared(requests, prefix, own):
    """Tables of requests with the same first blocks, in an order of their own, then blocks of their own."""
    rng = np.random.default_rng(prefix)
    first = rng.permutation(prefix)
    return [np.concatenate([first, prefix + r * own + np.arange(own)]) for r in range(requests)]


@pytest.mark.parametrize("fresh", [[1] * 24, [1, 3, 2, 6] * 6, [40, 1, 90, 17] * 6])
@pytest.mark.parametrize("block,dim,dtype", [(16, 128, BF), (32, 64, HF), (128, 96, BF)])
@pytest.mark.parametrize("window", [0, 700])
def test_a_prefix_that_all_requests_share(pp, fresh, block, dim, dtype, window):
    prefix, own = 1024 // block, -(-120 // block)
    length = [1024 + f + r % 20 for r, f in enumerate(fresh)]
    _compare(pp, _shared(len(fresh), prefix, own), fresh, length, 8, 2, dim, dtype, block, window)


@pytest.mark.parametrize("fresh", [[1] * 8, [50] * 8])
def test_a_tree_of_prefixes(pp, fresh):
    """Requests whose paths part one after another, and two that are the same in all blocks but the last."""
    depth, table, at = 10, [], 100
    for r in range(8):
        row = list(range(depth * 2)) if r == 0 else list(table[r - 1])
        for j in range(2 * depth - 2 * r, 2 * depth):
            row[j] = at
            at += 1
        table.append(row)
    last = np.arange(8)[:, None] + at
    table = np.concatenate([np.asarray(table), last, last + 8, last + 16, last + 24], 1)
    _compare(pp, table, fresh, [16 * 2 * depth + f for f in fresh], 4, 2, 64, BF, 16)


@pytest.mark.parametrize("fresh", [[1, 1], [60, 60]])
def test_a_block_twice_in_a_row(pp, fresh):
    """The same block at several places of a request's table is read at each of them."""
    _compare(pp, [[0, 1, 0, 2, 2, 3, 0, 4], [5, 5, 5, 5, 6, 1, 1, 7]], fresh, [128, 117], 4, 2, 64, HF, 16)


@pytest.mark.parametrize("heads,kv_heads", [(41, 1), (47, 1), (48, 1), (96, 2), (144, 3), (49, 1), (64, 1), (128, 2)])
@pytest.mark.parametrize("dim,dtype", [(128, BF), (64, HF)])
def test_single_tokens_of_wide_groups(pp, heads, kv_heads, dim, dtype):
    """Groups up to 48 without a workspace, wider ones with one."""
    length = [1, 17, 400, 1300, 64]
    at = np.arange(5 * 82).reshape(5, 82)
    _compare(pp, at, [1] * 5, length, heads, kv_heads, dim, dtype, 16)


def test_wide_groups_without_a_workspace_are_refused(pp):
    cache, exp = ref.to8(torch.randn((2, 16, 1, 64), device="cuda"))
    q = torch.zeros((1, 49, 64), dtype=BF, device="cuda")
    with pp.KVCache.like(cache) as kv:
        with pytest.raises(pp.PPError, match="workspace"):
            pp.pp_paged_attention8(kv, q, cache, exp, cache, exp.clone(), _i32([[0, 1]]), _i32([0, 1]), _i32([20]), 1, torch.empty_like(q), 0.1)
        kv.sync()


@pytest.mark.parametrize("e", [-39, -1, 0, 7, 39])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_the_border_of_a_scale(pp, e, dtype):
    """448 * 2^e has exponent e, the next number of the type e + 1 (bf16's is 450 * 2^e, f16's 448.25 * 2^e), and the one
    before it e."""
    step = 2.0 if dtype == BF else 0.25
    if dtype == HF and not -20 <= e <= 7:
        e = max(-20, min(7, e))
        step = max(step, 2.0 ** -24 / 2.0 ** e)             # f16's subnormal numbers
    for value, exponent in ((448.0 - step, e), (448.0, e), (448.0 + step, e + 1)):
        x = torch.zeros((1, 1, 16), dtype=dtype, device="cuda")
        x[0, 0, 3] = value * 2.0 ** e
        assert float(x[0, 0, 3]) == value * 2.0 ** e        # a number of the type
        code = [torch.zeros((1, 8, 1, 16), dtype=torch.float8_e4m3fn, device="cuda") for _ in range(2)]
        exp = [torch.zeros((1, 1), dtype=torch.int8, device="cuda") for _ in range(2)]
        with pp.KVCache.like(code[0], dtype=dtype) as kv:
            pp.pp_kv_write8(kv, x, -x, torch.zeros(1, dtype=torch.int64, device="cuda"), code[0], exp[0], code[1], exp[1])
            kv.sync()
        assert int(exp[0]) == int(exp[1]) == exponent
        assert float(code[0][0, 0, 0, 3].float()) == -float(code[1][0, 0, 0, 3].float()) == float(ref.e4m3(value * 2.0 ** (e - exponent)))
