"""pp_paged_attention8 against its 64-bit form (kv8_reference.py), at the sizes, layouts and masks
where it can go wrong, and its refusals.  The single-token kernel and that of chunks are both
reached at small sizes: max_q chooses between them and nothing else."""
import math

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


def _case(pp, fresh, cached, heads, kv_heads, dim, dtype=BF, block=16, window=0, order="token", seed=0, max_q=None,
          scale=None, spread=2.0, lse=True, pad=0, edit=None, room=0):
    """Runs the call and compares it with the 64-bit form within its bound.  Rows of the caches that hold no token are
    NaN, blocks that hold none have any exponents; table entries past a request's end are out of range."""
    torch.manual_seed(seed)
    rng = np.random.default_rng(seed)
    length = [max(0, f + c) for f, c in zip(fresh, cached)]
    need = [-(-n // block) for n in length]
    blocks = sum(need) + 3
    shape = (blocks, block, kv_heads, dim) if order == "token" else (blocks, kv_heads, block, dim)
    code, exp = [], []
    for i in range(2):
        x = torch.randn(shape, device="cuda")
        x = x if order == "token" else x.transpose(1, 2)
        x = x * torch.exp2(torch.randn((blocks, 1, kv_heads, 1), device="cuda") * (0.7 if i == 0 else 2.0))
        c, e = ref.to8(x)
        code.append(c)
        exp.append(e)
    order_ = rng.permutation(blocks)
    table = np.full((len(fresh), max(need + [1]) + 1), 1 << 30)
    bad = torch.ones((blocks, block), dtype=torch.bool, device="cuda")
    at = 0
    for r, n in enumerate(need):
        table[r, :n] = order_[at:at + n]
        at += n
        for x in range(n):
            bad[int(table[r, x]), :max(0, min(block, length[r] - x * block))] = False
    for c, e in zip(code, exp):
        c.view(torch.uint8)[bad] = 0x7f
        e[torch.tensor(order_[at:], device="cuda")] = 127
    tokens = sum(fresh)
    q = (torch.randn((tokens + pad, heads + 1, dim), device="cuda") * spread).to(dtype)[:, 1:]
    if pad:
        q[tokens:] = math.nan
    if edit:
        edit(q, code, exp, table)
    out = torch.full((tokens + pad, heads, dim), 7.0, dtype=dtype, device="cuda")
    lse_t = torch.full((tokens + pad, heads), 7.0, device="cuda") if lse else None
    q_start = np.concatenate([[0], np.cumsum(fresh)]).astype(np.int32)
    scale = dim ** -0.5 if scale is None else scale
    table_t = _i32(table)
    max_q = max(fresh + [0]) if max_q is None else max_q
    direct = max_q * (heads // kv_heads) <= 48
    with pp.KVCache.like(code[0], dtype=dtype) as kv:
        size = kv.workspace_size(len(fresh), table.shape[1], sum(need) + room)
        workspace = None if direct else torch.full((size,), 0x7f, dtype=torch.uint8, device="cuda")
        for _ in range(2):
            pp.pp_paged_attention8(kv, q, code[0], exp[0], code[1], exp[1], table_t, _i32(q_start), _i32(length), max_q, out,
                                   scale, window=window, lse=lse_t, workspace=workspace)
        kv.sync()
    want, wl, tol, ltol = ref.attention8(q[:tokens], code[0], exp[0], code[1], exp[1], table_t, q_start, length, scale,
                                         window, direct)
    nan = want.isnan()
    assert torch.equal(out[:tokens].isnan(), nan)
    err = (out[:tokens].double() - want).abs()[~nan]
    assert not (err > tol[~nan]).any() and not err.isnan().any(), \
        f"{int((~(err <= tol[~nan])).sum())} of {err.numel()} out of bound, worst {float((err / tol[~nan].clamp(min=1e-30)).max())}"
    if lse:
        known = ~(nan.any(-1) & wl.isnan()) & (wl != -math.inf)
        assert torch.equal(lse_t[:tokens] == -math.inf, wl == -math.inf)
        assert not ((lse_t[:tokens].double() - wl).abs() > ltol)[known].any()
        assert (lse_t[tokens:] == 7).all()
    assert (out[tokens:] == 7).all()
    return out, lse_t, want


HEADS = [(1, 1), (4, 4), (4, 2), (7, 1), (16, 2), (28, 4), (32, 2), (40, 1)]


@pytest.mark.parametrize("heads,kv_heads", HEADS)
@pytest.mark.parametrize("dim,dtype", [(128, BF), (64, HF), (80, BF), (16, HF), (112, HF), (48, BF)])
def test_single_tokens(pp, heads, kv_heads, dim, dtype):
    _case(pp, [1] * 9, [0, 1, 14, 15, 16, 63, 64, 127, 700], heads, kv_heads, dim, dtype)


@pytest.mark.parametrize("block", [8, 16, 32, 64, 128, 256, 512])
@pytest.mark.parametrize("order", ["token", "head"])
def test_single_tokens_blocks(pp, block, order):
    _case(pp, [1] * 5, [5, 255, 511, 512, 1030], 8, 2, 128, block=block, order=order)
    _case(pp, [1] * 5, [5, 255, 511, 512, 1030], 8, 2, 64, HF, block=block, order=order)


@pytest.mark.parametrize("window", [1, 2, 63, 64, 65, 300, 5000])
@pytest.mark.parametrize("fresh", [[1] * 5, [3, 1, 8, 5, 2]])
def test_few_tokens_window(pp, window, fresh):
    _case(pp, fresh, [0, 64, 300, 511, 1500], 8, 2, 64, window=window)


@pytest.mark.parametrize("requests,cached", [(1, 20_000), (2, 9001), (3, 1), (200, 130), (700, 3)])
def test_single_tokens_split(pp, requests, cached):
    rng = np.random.default_rng(requests)
    _case(pp, [1] * requests, [cached] + [int(x) for x in rng.integers(0, cached + 1, size=requests - 1)], 8, 2, 128)


@pytest.mark.parametrize("fresh", [[8, 1, 0, 5, 2], [0, 1, 0, 0, 1]])
def test_few_tokens_with_nan_past_the_end(pp, fresh):
    """Rows past a request's end lie in the tiles of rows that end before them."""
    _case(pp, fresh, [3, 9, 5, 123, 0], 8, 2, 128)
    _case(pp, fresh, [3, 9, 5, 123, 0], 8, 2, 64, block=8)


@pytest.mark.parametrize("max_q", [1, 9])
def test_max_q_chooses_the_kernel_and_nothing_else(pp, max_q):
    _case(pp, [5, 1, 0, 130], [0, 40, 7, 100], 8, 2, 128, max_q=max_q)


@pytest.mark.parametrize("heads,kv_heads", HEADS)
@pytest.mark.parametrize("dim,dtype", [(128, BF), (64, HF), (96, HF), (48, BF)])
def test_chunks(pp, heads, kv_heads, dim, dtype):
    _case(pp, [3, 1, 0, 65, 130], [0, 700, 5, 64, 131], heads, kv_heads, dim, dtype)


@pytest.mark.parametrize("block", [8, 16, 32, 64, 128, 256, 512])
@pytest.mark.parametrize("order", ["token", "head"])
def test_chunks_blocks(pp, block, order):
    _case(pp, [40, 260, 2], [5, 300, 1100], 4, 2, 128, block=block, order=order)


@pytest.mark.parametrize("window", [1, 2, 64, 127, 128, 129, 400, 5000])
@pytest.mark.parametrize("heads,kv_heads", [(2, 2), (8, 1)])
def test_chunks_window(pp, window, heads, kv_heads):
    _case(pp, [300, 33, 1], [0, 640, 900], heads, kv_heads, 64, window=window)


@pytest.mark.parametrize("requests,fresh,cached", [(1, 34, 20_000), (2, 40, 9000), (5, 100, 3000), (400, 12, 10)])
def test_chunks_split(pp, requests, fresh, cached):
    rng = np.random.default_rng(fresh)
    _case(pp, [fresh] + [int(x) for x in rng.integers(0, fresh + 1, size=requests - 1)],
          [cached] + [int(x) for x in rng.integers(0, cached + 1, size=requests - 1)], 8, 2, 128)


@pytest.mark.parametrize("fresh,cached", [([3, 8, 3], [-1, -3, -3]), ([40, 200, 3], [-10, -150, -3])])
def test_rows_that_see_nothing(pp, fresh, cached):
    out, lse, _ = _case(pp, fresh, cached, 8, 2, 64)
    n = -cached[0]
    assert int((out[:n] != 0).sum()) == 0 and (lse[:n] == -math.inf).all()


@pytest.mark.parametrize("dtype", [BF, HF])
def test_padded_step_without_lse(pp, dtype):
    _case(pp, [1, 1], [30, 200], 8, 2, 128, dtype, lse=False, pad=5)
    _case(pp, [9, 70], [30, 200], 8, 2, 128, dtype, lse=False, pad=200, room=50)


@pytest.mark.parametrize("fresh", [[1, 1], [64, 300]])
def test_sharp_and_flat_weights(pp, fresh):
    _case(pp, fresh, [900, 500], 8, 2, 128, scale=1.0, spread=3.0)
    _case(pp, fresh, [900, 500], 8, 2, 64, scale=1e-6)


@pytest.mark.parametrize("max_q", [1, 100])
@pytest.mark.parametrize("dim", [64, 128])
def test_scales_far_apart(pp, max_q, dim):
    """Blocks' values of sizes from 2^-40 to 2^40, with the weight on the small ones, on the large ones and on all."""
    for which, scale in ((0, 0.5), (1, 0.5), (None, 1e-3)):
        def edit(q, code, exp, table):
            span = torch.linspace(-40, 40, exp[1].shape[0], device="cuda").round().to(torch.int8)
            exp[1][:] = span[:, None]
            if which is not None:                           # keys of the small (0) or large (1) values point along q
                q[:] = 1.0
                low = (span < 0) == (which == 0)
                code[0].view(torch.uint8)[low] = 0x38       # 1.0
                code[0].view(torch.uint8)[~low] = 0xb8      # -1.0
                exp[0][:] = 0
        _case(pp, [1, 1, 1], [1000, 77, 350], 4, 1, dim, BF, max_q=max_q, scale=scale, edit=edit, block=8)


@pytest.mark.parametrize("max_q", [1, 100])
def test_keys_scales_far_apart(pp, max_q):
    def edit(q, code, exp, table):
        exp[0][:] = (torch.arange(exp[0].numel(), device="cuda") % 9 - 30).view(exp[0].shape).to(torch.int8)
    _case(pp, [1, 1], [1000, 77], 4, 2, 64, BF, max_q=max_q, scale=2.0 ** 18, edit=edit)


def test_exponents_outside_the_range_are_read_as_its_ends(pp):
    def edit(q, code, exp, table):
        exp[1][::3] = 100
        exp[1][1::3] = -100
    for max_q in (1, 100):
        _case(pp, [1, 1], [500, 77], 4, 2, 64, BF, max_q=max_q, edit=edit)


@pytest.mark.parametrize("dtype", [BF, HF])
def test_queries_of_any_size(pp, dtype):
    """A power of two a row: rows of zeros, of tiny and of the largest numbers, an infinity in one place."""
    def edit(q, code, exp, table):
        for i, f in enumerate((0.0, 2.0 ** -14, 2.0 ** -24, 200.0)):
            q[:, i] = (q[:, i].float() * f).to(dtype)
    _case(pp, [1, 4, 2], [300, 40, 7], 4, 2, 64, dtype, edit=edit)
    if dtype == BF:
        def far(q, code, exp, table):
            q[:, 0] *= 2.0 ** -100
            q[:, 1] *= 2.0 ** 100
        _case(pp, [1, 4, 2], [300, 40, 7], 4, 2, 64, dtype, edit=far, scale=2.0 ** -100)


@pytest.mark.parametrize("fresh", [[1], [6], [50]])
def test_nan_in_seen_rows(pp, fresh):
    """A NaN of V reaches the rows that see it, in its column, and no others; one of K makes a row NaN."""
    def v_edit(q, code, exp, table):
        code[1].view(torch.uint8)[int(table[0, 2]), 3, 1, 5] = 0xff
        code[1].view(torch.uint8)[int(table[0, (40 + fresh[0] - 1) // 16]), (40 + fresh[0] - 1) % 16, 0, 20] = 0x7f
    out, _, want = _case(pp, fresh, [40], 4, 2, 64, edit=v_edit, spread=0.1)
    assert out[-1, 0, 20].isnan() and int(out.isnan().sum()) == 2 * fresh[0] + 2

    def k_edit(q, code, exp, table):
        code[0].view(torch.uint8)[int(table[0, (40 + fresh[0] - 1) // 16]), (40 + fresh[0] - 1) % 16, 0, 20] = 0x7f
    out, _, _ = _case(pp, fresh, [40], 4, 2, 64, edit=k_edit)
    assert out[-1, :2].isnan().all() and not out[:-1].isnan().any() and not out[:, 2:].isnan().any()


def test_infinite_queries(pp):
    """All visible scores -infinity: 0 / 0, as the formula has it."""
    for max_q in (1, 100):
        for dtype in (BF, HF):
            q = torch.zeros((1, 1, 64), dtype=dtype, device="cuda")
            q[0, 0, 0] = -math.inf
            kc, ke = ref.to8(torch.rand((2, 16, 1, 64), device="cuda") + 1)
            out, lse = torch.zeros_like(q), torch.zeros((1, 1), device="cuda")
            with pp.KVCache.like(kc, dtype=dtype) as kv:
                w = torch.empty(kv.workspace_size(1, 2, 2), dtype=torch.uint8, device="cuda")
                pp.pp_paged_attention8(kv, q, kc, ke, kc, ke.clone(), _i32([[0, 1]]), _i32([0, 1]), _i32([20]), max_q, out, 0.1,
                                       lse=lse, workspace=w)
                kv.sync()
            # 0 * anything else is 0: the score is -infinity for every key
            assert out.isnan().all() and (lse == -math.inf).all()


def test_f16_of_large_and_small_values(pp):
    """Unpacked to f16, what it does not reach becomes its largest number; NaN stays."""
    kc = torch.zeros((1, 16, 1, 16), device="cuda")
    vc = torch.zeros((1, 16, 1, 16), device="cuda")
    vc[0, :, 0, 0], vc[0, :, 0, 1], vc[0, :, 0, 2], vc[0, :, 0, 3] = 448, -448, 1, math.nan
    code = [x.to(torch.float8_e4m3fn) for x in (kc, vc)]
    ke, ve = (torch.full((1, 1), e, dtype=torch.int8, device="cuda") for e in (0, 8))
    q = torch.ones((1, 1, 16), dtype=HF, device="cuda")
    out = torch.empty_like(q)
    with pp.KVCache.like(code[0], dtype=HF) as kv:
        w = torch.empty(kv.workspace_size(1, 1, 1), dtype=torch.uint8, device="cuda")
        pp.pp_paged_attention8(kv, q, code[0], ke, code[1], ve, _i32([[0]]), _i32([0, 1]), _i32([1]), 100, out, 1.0, workspace=w)
        kv.sync()
    assert out[0, 0, :3].tolist() == [65504.0, -65504.0, 256.0] and out[0, 0, 3].isnan() and (out[0, 0, 4:] == 0).all()


@pytest.mark.parametrize("max_q", [1, 100])
def test_bounds(pp, max_q):
    """Blocks out of range read as zeros, lengths and offsets are cut; all reported, none of it fatal."""
    kc, ke = ref.to8(torch.randn((4, 16, 2, 64), device="cuda"))
    vc, ve = ref.to8(torch.randn((4, 16, 2, 64), device="cuda"))
    q = torch.randn((2, 4, 64), device="cuda").to(BF)
    out = torch.empty_like(q)
    with pp.KVCache.like(kc) as kv:
        w = torch.empty(kv.workspace_size(2, 2, 4), dtype=torch.uint8, device="cuda")
        run = lambda table, q_start, length: pp.pp_paged_attention8(
            kv, q, kc, ke, vc, ve, _i32(table), _i32(q_start), _i32(length), max_q, out, 0.1, workspace=w)
        run([[0, 1], [2, 3]], [0, 1, 2], [20, 32])
        kv.sync()
        good = out.clone()
        for table, q_start, length in (([[0, 4], [2, 3]], [0, 1, 2], [20, 32]), ([[0, -1], [2, 3]], [0, 1, 2], [20, 32]),
                                       ([[0, 1 << 30], [2, 3]], [0, 1, 2], [20, 32]), ([[0, 1], [2, 3]], [0, 1, 2], [20, 33]),
                                       ([[0, 1], [2, 3]], [0, 1, 5], [20, 32]), ([[0, 1], [2, 3]], [-4, 1, 2], [20, 32]),
                                       ([[0, 1], [2, 3]], [0, 1, 2], [-3, 32])):
            run(table, q_start, length)
            with pytest.raises(pp.PPError, match="PP_EBOUNDS"):
                kv.sync()
            assert torch.equal(out[1], good[1]) and out.isfinite().all()
        run([[0, 1], [2, 3]], [0, 1, 2], [20, 32])
        kv.sync()
        assert torch.equal(out, good)


def test_a_workspace_that_is_too_small(pp):
    """Reported on the host where it has no room for a block, else on the device; what it has room for is right."""
    kc, ke = ref.to8(torch.randn((8, 16, 1, 64), device="cuda"))
    vc, ve = ref.to8(torch.randn((8, 16, 1, 64), device="cuda"))
    q = torch.randn((80, 1, 64), device="cuda").to(BF)
    table, q_start, length = _i32([[0, 1, 2, 3], [4, 5, 6, 7]]), _i32([0, 40, 80]), _i32([64, 64])
    with pp.KVCache.like(kc) as kv:
        def run(bytes_):
            out = torch.zeros_like(q)
            w = None if bytes_ is None else torch.empty(bytes_, dtype=torch.uint8, device="cuda")
            pp.pp_paged_attention8(kv, q, kc, ke, vc, ve, table, q_start, length, 100, out, 0.1, workspace=w)
            return out
        for bytes_ in (None, 0, 16, kv.workspace_size(2, 4, 1) - 1):
            with pytest.raises(pp.PPError, match="workspace"):
                run(bytes_)
        want = run(kv.workspace_size(2, 4, 8))
        kv.sync()
        for blocks in (1, 4, 7):
            got = run(kv.workspace_size(2, 4, blocks))
            with pytest.raises(pp.PPError, match="PP_EBOUNDS"):
                kv.sync()
            assert got.isfinite().all() and torch.equal(got[:40], want[:40]) == (blocks >= 4)
        with pytest.raises(pp.PPError, match="aligned"):
            w = torch.empty(kv.workspace_size(2, 4, 8) + 8, dtype=torch.uint8, device="cuda")[8:]
            pp.pp_paged_attention8(kv, q, kc, ke, vc, ve, table, q_start, length, 100, torch.zeros_like(q), 0.1, workspace=w)


def test_refusals(pp):
    kc, ke = ref.to8(torch.randn((4, 16, 2, 64), device="cuda"))
    vc, ve = ref.to8(torch.randn((4, 16, 2, 64), device="cuda"))
    base = torch.full((1 << 14,), 3.0, dtype=BF, device="cuda")
    q = torch.randn((5, 4, 64), device="cuda").to(BF)
    at = lambda first, *st: base.as_strided((5, 4, 64), (*st, 1), first)
    good = dict(q=q, k_cache=kc, k_exp=ke, v_cache=vc, v_exp=ve, block_table=_i32([[2, 0, 3]]), q_start=_i32([0, 5]),
                length=_i32([40]), max_q=5, out=at(0, 256, 64), scale=0.1)
    with pp.KVCache.like(kc) as kv:
        for bad in (dict(max_q=-1), dict(window=-1), dict(scale=0.0), dict(scale=math.nan), dict(out=at(0, 64, 64)),
                    dict(out=at(4, 256, 64)), dict(q=at(0, 260, 64)), dict(v_exp=ke),
                    dict(q=torch.zeros((5, 3, 64), dtype=BF, device="cuda"), out=torch.zeros((5, 3, 64), dtype=BF, device="cuda"))):
            with pytest.raises(pp.PPError, match="PP_EINVAL"):
                pp.pp_paged_attention8(kv, **{**good, **bad})
        with pytest.raises(ValueError, match="k_cache"):
            pp.pp_paged_attention(kv, q, torch.zeros((4, 16, 2, 64), dtype=BF, device="cuda"), vc, good["block_table"],
                                  good["q_start"], good["length"], 5, good["out"], 0.1)
        kv.sync()
        assert (base == 3).all()
    with pp.KVCache(4, 16, 2, 64) as kv:
        with pytest.raises(pp.PPError, match="16-bit"):
            kv.workspace_size(1, 1, 1)
        with pytest.raises(ValueError, match="eight_bit"):
            pp.pp_paged_attention8(kv, **good)


def test_nothing_to_do(pp):
    kc, ke = ref.to8(torch.randn((4, 16, 2, 64), device="cuda"))
    empty = torch.empty((0, 4, 64), dtype=BF, device="cuda")
    with pp.KVCache.like(kc) as kv:
        for requests in (0, 2):
            pp.pp_paged_attention8(kv, empty, kc, ke, kc, ke.clone(), torch.zeros((requests, 1), dtype=torch.int32, device="cuda"),
                                   _i32([0] * (requests + 1)), _i32([5] * requests), 1, empty, 0.1)
        kv.sync()


@pytest.mark.parametrize("fresh", [1, 50])
def test_graphs_and_streams(pp, fresh):
    """Captured, replayed after new rows and lengths; calls on another stream come after the last one's."""
    torch.manual_seed(5)
    kc, ke = ref.to8(torch.randn((64, 16, 2, 64), device="cuda"))
    vc, ve = ref.to8(torch.randn((64, 16, 2, 64), device="cuda"))
    q = torch.randn((2 * fresh, 4, 64), device="cuda").to(BF)
    table = _i32(np.arange(64).reshape(2, 32)[:, ::-1].copy())
    q_start, length = _i32([0, fresh, 2 * fresh]), _i32([300, 77])
    out, lse = torch.empty_like(q), torch.empty((2 * fresh, 4), device="cuda")
    with pp.KVCache.like(kc) as kv:
        w = torch.empty(kv.workspace_size(2, 32, 64), dtype=torch.uint8, device="cuda")

        def call(**kw):
            pp.pp_paged_attention8(kv, q, kc, ke, vc, ve, table, q_start, length, fresh, out, 0.125, lse=lse, workspace=w, **kw)

        def check():
            want, wl, tol, ltol = ref.attention8(q, kc, ke, vc, ve, table, q_start.tolist(), length.tolist(), 0.125, 0, fresh == 1)
            assert ((out.double() - want).abs() <= tol).all() and ((lse.double() - wl).abs() <= ltol).all()

        for stream in (torch.cuda.Stream(), torch.cuda.Stream(), None):
            if stream:
                stream.wait_stream(torch.cuda.current_stream())
            call(stream=stream)
        kv.sync()
        check()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        for step in range(3):
            q.copy_(torch.randn_like(q))
            length += 57
            graph.replay()
            kv.sync()
            check()


def test_two_handles_at_once(pp):
    """A handle and a workspace each: calls on two streams may overlap."""
    torch.manual_seed(6)
    kc, ke = ref.to8(torch.randn((256, 16, 2, 128), device="cuda"))
    vc, ve = ref.to8(torch.randn((256, 16, 2, 128), device="cuda"))
    table = _i32(np.arange(256)[None])
    handles = [pp.KVCache.like(kc) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    runs = []
    for i, fresh in enumerate((200, 1)):
        q = torch.randn((fresh, 8, 128), device="cuda").to(BF)
        w = torch.empty(handles[i].workspace_size(1, 256, 256), dtype=torch.uint8, device="cuda")
        out = torch.empty_like(q)
        runs.append((q, w, out, _i32([0, fresh]), _i32([4000 + i])))
    torch.cuda.synchronize()
    for _ in range(20):
        for kv, stream, (q, w, out, q_start, length) in zip(handles, streams, runs):
            pp.pp_paged_attention8(kv, q, kc, ke, vc, ve, table, q_start, length, len(q), out, 0.1, workspace=w, stream=stream)
    for kv, stream, (q, w, out, q_start, length) in zip(handles, streams, runs):
        kv.sync(stream)
        want, _, tol, _ = ref.attention8(q, kc, ke, vc, ve, table, q_start.tolist(), length.tolist(), 0.1, 0, len(q) == 1)
        assert ((out.double() - want).abs() <= tol).all()
        kv.close()


def test_a_cache_beyond_32_bits(pp):
    """Blocks whose codes lie more than 2^32 bytes into the cache."""
    blocks, block, heads, dim = 70_000, 128, 4, 128                      # 4.6e9 bytes each
    code = [torch.empty((blocks, block, heads, dim), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2)]
    exp = [torch.zeros((blocks, heads), dtype=torch.int8, device="cuda") for _ in range(2)]
    ids = [69_999, 3, 66_000, 34_000]
    slot = np.concatenate([i * block + np.arange(block) for i in ids])
    k, v = (torch.randn((512, heads, dim), device="cuda").to(BF) for _ in range(2))
    table, some = _i32([ids]), torch.tensor(ids, device="cuda")
    with pp.KVCache.like(code[0]) as kv:
        pp.pp_kv_write8(kv, k, v, torch.tensor(slot, device="cuda"), code[0], exp[0], code[1], exp[1])
        for fresh in (1, 60):
            q = torch.randn((fresh, 8, dim), device="cuda").to(BF)
            out = torch.empty_like(q)
            w = torch.empty(kv.workspace_size(1, 4, 4), dtype=torch.uint8, device="cuda")
            pp.pp_paged_attention8(kv, q, code[0], exp[0], code[1], exp[1], table, _i32([0, fresh]), _i32([512]), fresh, out, 0.1,
                                   workspace=w)
            kv.sync()
            small = [c.view(torch.uint8)[some].view(torch.float8_e4m3fn) for c in code]
            for x, c, e in zip((k, v), small, exp):
                want = x.double().view(4, block, heads, dim)
                got = ref.scaled(c, e[some])
                assert ((got - want).abs() <= torch.maximum(2.0 ** -4 * want.abs(), 2.0 ** -10 * torch.exp2(e[some].double())[:, None, :, None])).all()
            want, _, tol, _ = ref.attention8(q, small[0], exp[0][some], small[1], exp[1][some], _i32([[0, 1, 2, 3]]), [0, fresh],
                                             [512], 0.1, 0, fresh == 1)
            assert ((out.double() - want).abs() <= tol).all()
