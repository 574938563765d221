"""The paged cache's operators against plain 64-bit forms (kv_reference.py), at
the sizes, layouts and masks where they can go wrong, and their refusals."""
import math

import numpy as np
import pytest

from tests import kv_reference as ref
from tests.test_kv_host import _closed, _forest, _walk

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


# ---------------------------------------------------------------------------
# block tables
# ---------------------------------------------------------------------------
def _tables_case(seed, requests, admitted, block, chunks, longest, per, pad):
    rng = np.random.default_rng(seed)
    parent = _forest(rng, chunks, 0.8)
    weight = rng.integers(1, 3, size=chunks).astype(np.int32)
    res = _closed(rng, parent, 0.9)
    return rng, parent, weight, res


@pytest.mark.parametrize("requests,admitted,block,chunks,longest,per,pad", [
    (1, 0, 16, 1, 1, 1, 0), (1, 1, 8, 3, 40, 2, 5), (7, 3, 16, 50, 100, 4, 0), (33, 33, 32, 200, 300, 16, 63),
    (300, 100, 16, 500, 700, 32, 1), (1500, 700, 64, 2000, 90, 8, 0), (5000, 0, 512, 1, 30, 1, 0)])
def test_block_tables(pp, requests, admitted, block, chunks, longest, per, pad):
    rng, parent, weight, res = _tables_case(requests, requests, admitted, block, chunks, longest, per, pad)
    rec, used = pp.pp_chunk_map(parent, weight, res, per)
    node = np.full(requests, -1)
    node[rng.permutation(requests)[:admitted]] = rng.integers(0, chunks, size=admitted)
    path = lambda v: np.array(_walk(rec, v)[0], np.int64)
    length, cached = np.zeros(requests, np.int64), np.zeros(requests, np.int64)
    for r in range(requests):
        if node[r] >= 0:
            # shorter than the prefix, its exact end, one more, longer; and empty
            n = len(path(int(node[r]))) * block
            length[r] = max(0, n + rng.choice([-1 - n // 2, -n, 0, 1, int(rng.integers(1, longest + 1))]))
            cached[r] = rng.integers(-5, 99)                # not read
        else:
            length[r] = rng.integers(0, longest + 1)
            cached[r] = rng.integers(0, length[r] + 1)
    c = np.where(node < 0, cached, 0)
    held = -(-c // block)
    need = -(-length // block)
    total = used + int(held.sum()) + int(need.sum()) + 4
    other = rng.permutation(np.arange(used, total))
    width = int(need.max()) + 1
    table = np.full((requests, width), -7)
    at = 0
    for r in np.flatnonzero(node < 0):
        table[r, :held[r]] = other[at:at + held[r]]
        at += held[r]
    free = other[at:]
    want = ref.block_tables(length, cached, node, path, table, free, 1, block, 0)
    capacity = len(want[1]) + pad
    want = ref.block_tables(length, cached, node, path, table, free, 1, block, capacity)
    t = dict(table=_i32(table), slot=torch.full((capacity,), 5, device="cuda"), pos=_i32(np.full(capacity, 5)),
             q=_i32(np.zeros(requests + 1)), out=_i32([0]))
    with pp.KVCache(total, block, 1, 8) as kv:
        for _ in range(2):                                  # the same again: nothing is kept
            pp.pp_block_tables(kv, _i32(length), _i32(cached), t["table"], t["slot"], t["pos"], t["q"], _i32(free),
                               _i32([1]), t["out"], node=_i32(node), chunk_map=_i32(rec))
            kv.sync()
            for got, exp in zip((t["table"], t["slot"], t["pos"], t["q"], t["out"][0]), want):
                assert np.array_equal(got.cpu().numpy(), exp)


def test_block_tables_without_requests_or_tokens(pp):
    empty = _i32([])
    with pp.KVCache(4, 16, 1, 8) as kv:
        slot, pos, q, out = torch.zeros(3, dtype=torch.int64, device="cuda"), _i32([9, 9, 9]), _i32([7]), _i32([0])
        pp.pp_block_tables(kv, empty, empty, torch.zeros((0, 1), dtype=torch.int32, device="cuda"), slot, pos, q,
                           empty, _i32([0]), out)
        kv.sync()
        assert slot.tolist() == [-1] * 3 and pos.tolist() == [0] * 3 and q.tolist() == [0] and out.tolist() == [0]


@pytest.mark.parametrize("change,slots", [
    (dict(length=[-1, 3]), [-1] * 4), (dict(length=[33, 3]), None), (dict(cached=[3, 3]), [-1] * 4),
    (dict(cached=[-1, 3]), None), (dict(free=[9]), [-1] * 4), (dict(free=[]), [-1] * 4),
    (dict(node=[5, -1]), None), (dict(node=[-2, -1]), None), (dict(head=[2]), [-1] * 4),
    (dict(head=[-1]), None), (dict(table=-1, length=[2, 4]), None),
])
def test_block_tables_reports_bounds(pp, change, slots):
    """Values in device memory that are out of range: reported, and nothing outside the buffers is touched."""
    a = dict(length=[2, 3], cached=[0, 3], node=None, free=[3, 2], head=[0], table=1)
    a.update(change)
    with pp.KVCache(4, 16, 1, 8) as kv:
        table = torch.full((2, 2), a["table"], dtype=torch.int32, device="cuda")
        slot, pos = torch.zeros(4, dtype=torch.int64, device="cuda"), _i32([0] * 4)
        q, out = _i32([0] * 3), _i32([0])
        extra = {} if a["node"] is None else dict(node=_i32(a["node"]), chunk_map=_i32([[-1, 0, 0, 1]]))
        pp.pp_block_tables(kv, _i32(a["length"]), _i32(a["cached"]), table, slot, pos, q, _i32(a["free"]),
                           _i32(a["head"]), out, **extra)
        with pytest.raises(pp.PPError, match="PP_EBOUNDS"):
            kv.sync()
        kv.sync()                                            # read and cleared
        assert int(slot.max()) < 4 * 16 and int(out[0]) <= max(len(a["free"]), 0)
        if slots is not None:
            assert all(s in (-1,) for s in slot.tolist())


def test_block_tables_more_tokens_than_capacity(pp):
    with pp.KVCache(8, 16, 1, 8) as kv:
        buf = torch.full((6,), 77, dtype=torch.int64, device="cuda")
        slot, pos, q, out = buf[:4], _i32([0] * 4), _i32([0] * 3), _i32([0])
        pp.pp_block_tables(kv, _i32([3, 3]), _i32([0, 0]), _i32([[0], [0]]), slot, pos, q, _i32([6, 5]), _i32([0]), out)
        with pytest.raises(pp.PPError, match="PP_EBOUNDS"):
            kv.sync()
        assert buf.tolist() == [96, 97, 98, 80, 77, 77]


# ---------------------------------------------------------------------------
# writes
# ---------------------------------------------------------------------------
def _cache(blocks, block, heads, dim, dtype, order):
    shape = (blocks, block, heads, dim) if order == "token" else (blocks, heads, block, dim)
    t = torch.randn(shape, device="cuda").to(dtype)
    return t if order == "token" else t.transpose(1, 2)


@pytest.mark.parametrize("tokens,heads,dim,dtype,block,order", [
    (0, 2, 64, torch.bfloat16, 16, "token"), (1, 1, 8, torch.float16, 8, "token"),
    (77, 3, 80, torch.float16, 32, "head"), (1000, 8, 128, torch.bfloat16, 16, "token"),
    (513, 5, 96, torch.bfloat16, 512, "head"), (3, 300, 128, torch.float16, 8, "token")])
def test_write(pp, tokens, heads, dim, dtype, block, order):
    torch.manual_seed(tokens)
    blocks = tokens // block + 3
    kc, vc = (_cache(blocks, block, heads, dim, dtype, order) for _ in range(2))
    qkv = torch.randn((tokens, 2 * heads * dim + 8), device="cuda").to(dtype)
    k = qkv[:, 8:8 + heads * dim].unflatten(1, (heads, dim))
    v = qkv[:, 8 + heads * dim:].unflatten(1, (heads, dim)).flip(1).clone() if tokens % 2 else \
        qkv[:, 8 + heads * dim:].unflatten(1, (heads, dim))
    slot = torch.randperm(blocks * block, device="cuda")[:tokens]
    slot[::5] = -1 - slot[::5]
    ek, ev = kc.clone(), vc.clone()
    keep = slot >= 0
    ek[slot[keep] // block, slot[keep] % block] = k[keep]
    ev[slot[keep] // block, slot[keep] % block] = v[keep]
    with pp.KVCache.like(kc) as kv:
        pp.pp_kv_write(kv, k, v, slot, kc, vc)
        kv.sync()
    assert torch.equal(kc.view(torch.int16), ek.view(torch.int16))
    assert torch.equal(vc.view(torch.int16), ev.view(torch.int16))


def test_write_reports_bounds(pp):
    kc, vc = (torch.zeros((2, 8, 1, 8), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    rows = torch.ones((3, 1, 8), dtype=torch.bfloat16, device="cuda")
    with pp.KVCache.like(kc) as kv:
        pp.pp_kv_write(kv, rows, rows, torch.tensor([16, 3, 1 << 40], device="cuda"), kc, vc)
        with pytest.raises(pp.PPError, match="PP_EBOUNDS"):
            kv.sync()
    assert int(kc.sum()) == 8 and int(kc[0, 3].sum()) == 8 and int(vc.sum()) == 8


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------
def _attention_case(pp, fresh, cached, heads, kv_heads, dim, dtype=torch.bfloat16, block=16, window=0, order="token",
                    seed=0, max_q=None, poison=True, scale=None, spread=2.0, lse=True, pad=0, kc=None, vc=None):
    """Runs the kernel and compares it with the 64-bit form within its bound.
    Rows of the cache that hold no token are NaN and infinite; so are the padded rows of q."""
    torch.manual_seed(seed)
    rng = np.random.default_rng(seed)
    length = [max(0, f + c) for f, c in zip(fresh, cached)]
    need = [-(-n // block) for n in length]
    if kc is None:
        blocks = sum(need) + 3
        kc, vc = (_cache(blocks, block, kv_heads, dim, dtype, order) for _ in range(2))
        order_ = rng.permutation(blocks)
    else:
        blocks = kc.shape[0]
        order_ = rng.permutation(blocks)
    table = np.full((len(fresh), max(need + [1]) + 1), 1 << 30)          # entries past a request's end are not read
    at = 0
    bad = torch.ones((blocks, block), dtype=torch.bool, device="cuda")
    for r, n in enumerate(need):
        table[r, :n] = order_[at:at + n]
        at += n
        for x in range(n):
            bad[int(table[r, x]), :max(0, min(block, length[r] - x * block))] = False
    if poison:
        kc[bad] = float("nan")
        vc[bad] = float("inf")
    tokens = sum(fresh)
    q = (torch.randn((tokens + pad, heads + 1, dim), device="cuda") * spread).to(dtype)[:, 1:]
    if pad:
        q[tokens:] = float("nan")
    out = torch.full((tokens + pad, heads, dim), 7.0, dtype=dtype, device="cuda")
    lse_t = torch.full((tokens + pad, heads), 7.0, device="cuda") if lse else None
    q_start = np.concatenate([[0], np.cumsum(fresh)]).astype(np.int32)
    scale = dim ** -0.5 if scale is None else scale
    table_t = _i32(table)
    with pp.KVCache.like(kc) as kv:
        for _ in range(2):
            pp.pp_paged_attention(kv, q, kc, vc, table_t, _i32(q_start), _i32(length),
                                  max(fresh + [0]) if max_q is None else max_q, out, scale, window=window, lse=lse_t)
        kv.sync()
    want, wl, tol, ltol = ref.attention(q[:tokens], kc, vc, table_t, q_start, length, scale, window)
    err = (out[:tokens].double() - want).abs()
    assert not (err > tol).any() and not err.isnan().any(), \
        f"{int((~(err <= tol)).sum())} of {err.numel()} out of bound, worst {float((err / tol.clamp(min=1e-30)).max())}"
    if lse:
        empty = wl == -math.inf
        assert torch.equal(lse_t[:tokens] == -math.inf, empty)
        assert not ((lse_t[:tokens].double() - wl).abs() > ltol)[~empty].any()
        assert (lse_t[tokens:] == 7).all()
    assert (out[tokens:] == 7).all()
    return out


HEADS = [(1, 1), (4, 4), (4, 2), (7, 1), (16, 2), (28, 4), (32, 2), (40, 1)]


@pytest.mark.parametrize("heads,kv_heads", HEADS)
@pytest.mark.parametrize("dim,dtype", [(128, torch.bfloat16), (64, torch.float16), (80, torch.bfloat16),
                                       (8, torch.float16)])
def test_single_tokens(pp, heads, kv_heads, dim, dtype):
    _attention_case(pp, [1] * 9, [0, 1, 14, 15, 16, 63, 64, 127, 700], heads, kv_heads, dim, dtype)


@pytest.mark.parametrize("block", [8, 16, 32, 64, 128, 256, 512])
@pytest.mark.parametrize("order", ["token", "head"])
def test_single_tokens_blocks(pp, block, order):
    _attention_case(pp, [1] * 5, [5, 255, 511, 512, 1030], 8, 2, 128, block=block, order=order)


@pytest.mark.parametrize("window", [1, 2, 63, 64, 65, 300, 5000])
def test_single_tokens_window(pp, window):
    _attention_case(pp, [1] * 5, [0, 64, 300, 511, 1500], 8, 2, 64, window=window)


@pytest.mark.parametrize("requests,cached", [(1, 20_000), (2, 9001), (3, 1), (200, 130), (700, 3)])
def test_single_tokens_split(pp, requests, cached):
    """From one long context, split over all SMs and joined, to more requests than SMs."""
    rng = np.random.default_rng(requests)
    _attention_case(pp, [1] * requests, [cached] + [int(x) for x in rng.integers(0, cached + 1, size=requests - 1)],
                    8, 2, 128)


def test_single_tokens_some_without_any(pp):
    """Requests without new tokens, without tokens at all, and between others."""
    _attention_case(pp, [0, 1, 0, 0, 1, 1, 0], [5, 0, 0, 300, 0, 40, 0], 8, 4, 64)


def test_single_token_kernel_on_chunks(pp):
    """max_q chooses the kernel and nothing else."""
    _attention_case(pp, [5, 1, 0, 130], [0, 40, 7, 100], 8, 2, 128, max_q=1)
    _attention_case(pp, [1, 1, 1], [0, 40, 700], 8, 2, 128, max_q=9)


@pytest.mark.parametrize("heads,kv_heads", HEADS)
@pytest.mark.parametrize("dim,dtype", [(128, torch.bfloat16), (64, torch.float16), (96, torch.float16),
                                       (40, torch.bfloat16)])
def test_chunks(pp, heads, kv_heads, dim, dtype):
    _attention_case(pp, [3, 1, 0, 65, 130], [0, 700, 5, 64, 131], heads, kv_heads, dim, dtype)


@pytest.mark.parametrize("block", [8, 16, 32, 64, 128, 256, 512])
@pytest.mark.parametrize("order", ["token", "head"])
def test_chunks_blocks(pp, block, order):
    _attention_case(pp, [40, 260, 2], [5, 300, 1100], 4, 2, 128, block=block, order=order)


@pytest.mark.parametrize("window", [1, 2, 64, 127, 128, 129, 400, 5000])
@pytest.mark.parametrize("heads,kv_heads", [(2, 2), (8, 1)])
def test_chunks_window(pp, window, heads, kv_heads):
    _attention_case(pp, [300, 33, 1], [0, 640, 900], heads, kv_heads, 64, window=window)


@pytest.mark.parametrize("fresh,cached", [([1], [0]), ([2], [0]), ([127], [0]), ([128], [0]), ([129], [0]),
                                          ([255], [1]), ([256], [0]), ([257], [127]), ([513], [512])])
def test_chunks_lengths(pp, fresh, cached):
    _attention_case(pp, fresh, cached, 1, 1, 128, max_q=600)


@pytest.mark.parametrize("requests,fresh,cached", [(1, 16, 20_000), (2, 40, 9000), (5, 100, 3000), (400, 4, 10)])
def test_chunks_split(pp, requests, fresh, cached):
    rng = np.random.default_rng(fresh)
    _attention_case(pp, [fresh] + [int(x) for x in rng.integers(0, fresh + 1, size=requests - 1)],
                    [cached] + [int(x) for x in rng.integers(0, cached + 1, size=requests - 1)], 8, 2, 128)


def test_rows_that_see_nothing(pp):
    """Fewer tokens than queries: the first queries stand before the first key."""
    out = _attention_case(pp, [40, 200, 3], [-10, -150, -3], 8, 2, 64)
    assert int((out[:10] != 0).sum()) == 0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_padded_step_without_lse(pp, dtype):
    _attention_case(pp, [1, 1], [30, 200], 8, 2, 128, dtype, lse=False, pad=5)
    _attention_case(pp, [9, 70], [30, 200], 8, 2, 128, dtype, lse=False, pad=200)


@pytest.mark.parametrize("fresh", [[1, 1], [64, 300]])
def test_sharp_and_flat_weights(pp, fresh):
    """Large scores: the running maximum moves by more than any fixed step; tiny scores: all weights alike."""
    _attention_case(pp, fresh, [900, 500], 8, 2, 128, scale=1.0, spread=3.0)
    _attention_case(pp, fresh, [900, 500], 8, 2, 64, scale=1e-6)


def test_scores_that_grow_along_the_context(pp):
    """Every tile raises the maximum: the rescale runs in each."""
    torch.manual_seed(1)
    for fresh in ([1], [200]):
        n = 1000 + fresh[0]
        blocks = -(-n // 16)
        kc = torch.randn((blocks, 16, 1, 64), device="cuda").to(torch.bfloat16)
        vc = torch.randn_like(kc)
        q = torch.ones((fresh[0], 4, 64), dtype=torch.bfloat16, device="cuda")
        kc.view(-1, 64)[:] += (torch.arange(blocks * 16, device="cuda")[:, None] * 0.02).to(torch.bfloat16)
        table = torch.arange(blocks, dtype=torch.int32, device="cuda")[None]
        out = torch.empty_like(q)
        with pp.KVCache.like(kc) as kv:
            pp.pp_paged_attention(kv, q, kc, vc, table, _i32([0, fresh[0]]), _i32([n]), fresh[0], out, 0.125)
            kv.sync()
        want, _, tol, _ = ref.attention(q, kc, vc, table, [0, fresh[0]], [n], 0.125, 0)
        assert not ((out.double() - want).abs() > tol).any()


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("fresh,row", [([1], 200), ([300], 430), ([300], 150), ([40], 201)])
@pytest.mark.parametrize("window", [0, 60])
def test_values_out_of_range_stay_with_those_who_see_them(pp, bad, fresh, row, window):
    """An infinite or NaN V row changes exactly the queries that see it: in its own column only."""
    torch.manual_seed(3)
    n = 201 + fresh[0]
    blocks = -(-n // 16)
    kc, vc = (torch.randn((blocks, 16, 2, 64), device="cuda").to(torch.bfloat16) for _ in range(2))
    q = torch.randn((fresh[0], 6, 64), device="cuda").to(torch.bfloat16)
    table = torch.arange(blocks, dtype=torch.int32, device="cuda")[None]
    out, clean = torch.empty_like(q), torch.empty_like(q)
    with pp.KVCache.like(kc) as kv:
        pp.pp_paged_attention(kv, q, kc, vc, table, _i32([0, fresh[0]]), _i32([n]), fresh[0], clean, 0.125, window=window)
        vc[row // 16, row % 16, 1, 5] = bad
        pp.pp_paged_attention(kv, q, kc, vc, table, _i32([0, fresh[0]]), _i32([n]), fresh[0], out, 0.125, window=window)
        kv.sync()
    pos = torch.arange(n - fresh[0], n, device="cuda")
    sees = (pos >= row) & ((pos - row < window) if window else True)
    hit = torch.zeros(out.shape, dtype=torch.bool, device="cuda")
    hit[sees, 3:, 5] = True
    assert torch.equal(out[~hit], clean[~hit])
    if math.isnan(bad):
        assert out[hit].isnan().all()
    else:
        assert (out[hit] == bad).all()


@pytest.mark.parametrize("fresh,row", [([1], 100), ([300], 430), ([300], 150)])
def test_a_nan_key_stays_with_those_who_see_it(pp, fresh, row):
    torch.manual_seed(4)
    n = 201 + fresh[0]
    blocks = -(-n // 16)
    kc, vc = (torch.randn((blocks, 16, 1, 64), device="cuda").to(torch.float16) for _ in range(2))
    q = torch.randn((fresh[0], 3, 64), device="cuda").to(torch.float16)
    table = torch.arange(blocks, dtype=torch.int32, device="cuda")[None]
    out, clean = torch.empty_like(q), torch.empty_like(q)
    with pp.KVCache.like(kc) as kv:
        pp.pp_paged_attention(kv, q, kc, vc, table, _i32([0, fresh[0]]), _i32([n]), fresh[0], clean, 0.125)
        kc[row // 16, row % 16, 0, 5] = float("nan")
        pp.pp_paged_attention(kv, q, kc, vc, table, _i32([0, fresh[0]]), _i32([n]), fresh[0], out, 0.125)
        kv.sync()
    sees = torch.arange(n - fresh[0], n, device="cuda") >= row
    assert torch.equal(out[~sees], clean[~sees]) and out[sees].isnan().all()


@pytest.mark.parametrize("fresh", [[1, 1], [30, 70]])
def test_offsets_past_32_bits(pp, fresh):
    """Blocks 2^30 elements apart: offsets in elements pass 2^32."""
    base = torch.empty(4 * (1 << 30) + 16 * 2 * 64, dtype=torch.bfloat16, device="cuda")
    kc = base.as_strided((5, 16, 2, 64), (1 << 30, 128, 64, 1))
    base2 = torch.empty_like(base)
    vc = base2.as_strided((5, 16, 2, 64), (1 << 30, 128, 64, 1))
    kc.normal_()
    vc.normal_()
    _attention_case(pp, fresh, [32 - f for f in fresh], 8, 2, 64, kc=kc, vc=vc, poison=False) if fresh[0] == 1 else \
        _attention_case(pp, [30], [50], 8, 2, 64, kc=kc, vc=vc, poison=False)
    rows = torch.ones((2, 2, 64), dtype=torch.bfloat16, device="cuda")
    with pp.KVCache.like(kc) as kv:
        pp.pp_kv_write(kv, rows, rows * 2, torch.tensor([4 * 16 + 3, 2], device="cuda"), kc, vc)
        kv.sync()
    assert (kc[4, 3] == 1).all() and (vc[4, 3] == 2).all() and (kc[0, 2] == 1).all()


@pytest.mark.parametrize("max_q", [1, 100])
@pytest.mark.parametrize("change", [dict(table=[[0, 4, 2]]), dict(table=[[0, -1, 2]]), dict(length=[-3]),
                                    dict(length=[49]), dict(q_start=[0, 9]), dict(q_start=[0, -2]),
                                    dict(q_start=[-1, 5])])
def test_attention_reports_bounds(pp, max_q, change):
    a = dict(table=[[0, 1, 2]], length=[40], q_start=[0, 5])
    a.update(change)
    kc, vc = (torch.randn((4, 16, 1, 64), device="cuda").to(torch.bfloat16) for _ in range(2))
    q = torch.randn((5, 2, 64), device="cuda").to(torch.bfloat16)
    buf = torch.zeros((9, 2, 64), dtype=torch.bfloat16, device="cuda")
    with pp.KVCache.like(kc) as kv:
        pp.pp_paged_attention(kv, q, kc, vc, _i32(a["table"]), _i32(a["q_start"]), _i32(a["length"]), max_q, buf[2:7],
                              0.125)
        with pytest.raises(pp.PPError, match="PP_EBOUNDS"):
            kv.sync()
        kv.sync()
    assert not buf[:2].any() and not buf[7:].any() and not buf.isnan().any()


def test_stream_and_graph(pp):
    """A step (write, attention) on a side stream, then captured and replayed with new values."""
    torch.manual_seed(5)
    kc, vc = (torch.zeros((40, 16, 2, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    kc.normal_()
    vc.normal_()
    table = _i32(np.arange(40).reshape(2, 20))
    lens, q_start = _i32([300, 77]), _i32([0, 1, 2])
    q = torch.randn((2, 8, 128), device="cuda").to(torch.bfloat16)
    k, v = (torch.randn((2, 2, 128), device="cuda").to(torch.bfloat16) for _ in range(2))
    slot = torch.tensor([299, 20 * 16 + 76], device="cuda")
    out = torch.empty_like(q)
    side = torch.cuda.Stream()
    with pp.KVCache.like(kc) as kv:
        def step(stream):
            pp.pp_kv_write(kv, k, v, slot, kc, vc, stream=stream)
            pp.pp_paged_attention(kv, q, kc, vc, table, q_start, lens, 1, out, 0.09, stream=stream)
        side.wait_stream(torch.cuda.current_stream())
        step(side)
        torch.cuda.current_stream().wait_stream(side)
        first = out.clone()
        want, _, tol, _ = ref.attention(q, kc, vc, table, [0, 1, 2], [300, 77], 0.09, 0)
        assert not ((first.double() - want).abs() > tol).any()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(torch.cuda.current_stream())
        lens.copy_(_i32([299, 70]))
        q.mul_(0.5)
        for _ in range(3):
            graph.replay()
        kv.sync()
        want, _, tol, _ = ref.attention(q, kc, vc, table, [0, 1, 2], [299, 70], 0.09, 0)
        assert not ((out.double() - want).abs() > tol).any()


def test_refusals(pp):
    kc, vc = (torch.zeros((4, 16, 2, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q = torch.zeros((2, 4, 64), dtype=torch.bfloat16, device="cuda")
    table, q_start, lens = _i32([[0, 1]]), _i32([0, 2]), _i32([5])
    ok = dict(q=q, k_cache=kc, v_cache=vc, block_table=table, q_start=q_start, length=lens, max_q=2,
              out=torch.zeros_like(q), scale=0.1)
    with pp.KVCache.like(kc) as kv:
        pp.pp_paged_attention(kv, **ok)
        for bad in (dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")),
                    dict(window=-1), dict(max_q=-1),
                    dict(q=q[:, :3], out=torch.zeros_like(q[:, :3]))):
            with pytest.raises(pp.PPError, match="PP_EINVAL"):
                pp.pp_paged_attention(kv, **{**ok, **bad})
        odd = torch.zeros(2 * 4 * 64 + 1, dtype=torch.bfloat16, device="cuda")[1:].view(2, 4, 64)
        with pytest.raises(pp.PPError, match="aligned"):
            pp.pp_paged_attention(kv, **{**ok, "q": odd})
        skew = torch.zeros((2, 4, 65), dtype=torch.bfloat16, device="cuda")[:, :, :64]
        with pytest.raises(pp.PPError, match="strides"):
            pp.pp_paged_attention(kv, **{**ok, "q": skew})
        for bad in (dict(q=q.half()), dict(k_cache=kc[:3]), dict(k_cache=kc.transpose(1, 2)), dict(q_start=lens),
                    dict(length=lens.long()), dict(block_table=table[0]), dict(lse=torch.zeros(8, device="cuda")),
                    dict(out=torch.zeros((2, 4, 32), dtype=torch.bfloat16, device="cuda")),
                    dict(block_table=torch.zeros((1, 4), dtype=torch.int32, device="cuda")[:, ::2])):
            with pytest.raises(ValueError):
                pp.pp_paged_attention(kv, **{**ok, **bad})
        k = torch.zeros((2, 2, 64), dtype=torch.bfloat16, device="cuda")
        slot = torch.zeros(2, dtype=torch.int64, device="cuda")
        with pytest.raises(ValueError):
            pp.pp_kv_write(kv, k, k[:1], slot, kc, vc)
        with pytest.raises(ValueError):
            pp.pp_kv_write(kv, k, k, slot.int(), kc, vc)
        head = _i32([0])
        tab = dict(length=lens, cached=_i32([4]), block_table=table, slot_map=slot, position=_i32([0, 0]),
                   q_start=_i32([0, 0]), free_blocks=_i32([3]), free_head=head, free_head_out=_i32([0]))
        pp.pp_block_tables(kv, **tab)
        with pytest.raises(pp.PPError, match="different words"):
            pp.pp_block_tables(kv, **{**tab, "free_head_out": head})
        with pytest.raises(ValueError):
            pp.pp_block_tables(kv, **tab, node=_i32([0]))
        with pytest.raises(ValueError):
            pp.pp_block_tables(kv, **{**tab, "position": _i32([0])})
        many = torch.zeros(16385, dtype=torch.int32, device="cuda")
        with pytest.raises(pp.PPError, match="16384"):
            pp.pp_block_tables(kv, **{**tab, "length": many, "cached": many, "q_start": _i32(np.zeros(16386)),
                                      "block_table": torch.zeros((16385, 1), dtype=torch.int32, device="cuda")})
        kv.sync()
    with pytest.raises(RuntimeError):
        pp.pp_paged_attention(kv, **ok)


@pytest.mark.parametrize("fresh", [[1, 1, 1], [70, 1, 140]])
@pytest.mark.parametrize("dim,lead", [(128, 8), (64, 16), (72, 8)])
def test_output_in_a_wider_buffer(pp, fresh, dim, lead):
    """Output rows inside rows of another buffer, at 16-byte boundaries that are and are not 32-byte ones."""
    torch.manual_seed(6)
    length = [f + 90 for f in fresh]
    blocks = sum(-(-n // 16) for n in length)
    kc, vc = (torch.randn((blocks, 16, 2, dim), device="cuda").to(torch.bfloat16) for _ in range(2))
    table, at = np.zeros((3, 20)), 0
    for r, n in enumerate(length):
        table[r, :-(-n // 16)] = np.arange(at, at - (-n // 16))
        at -= -n // 16
    table = _i32(table)
    q = torch.randn((sum(fresh), 6, dim), device="cuda").to(torch.bfloat16)
    buf = torch.full((sum(fresh), 6 * dim + 2 * lead), 3.0, dtype=torch.bfloat16, device="cuda")
    out = buf[:, lead:-lead].unflatten(1, (6, dim))
    q_start = np.concatenate([[0], np.cumsum(fresh)])
    with pp.KVCache.like(kc) as kv:
        pp.pp_paged_attention(kv, q, kc, vc, table, _i32(q_start), _i32(length), max(fresh), out, dim ** -0.5)
        kv.sync()
    want, _, tol, _ = ref.attention(q, kc, vc, table, q_start, length, dim ** -0.5, 0)
    assert not ((out.double() - want).abs() > tol).any()
    assert (buf[:, :lead] == 3).all() and (buf[:, -lead:] == 3).all()


def test_many_requests_of_chunks(pp):
    """More requests than the kernel has threads, most of them small."""
    rng = np.random.default_rng(9)
    _attention_case(pp, [int(x) for x in rng.integers(0, 6, size=1100)], [int(x) for x in rng.integers(0, 60, size=1100)],
                    4, 2, 64, seed=9)


@pytest.mark.parametrize("fresh", [[1, 1, 1, 1], [90, 200, 3, 1]])
def test_a_query_out_of_range_stays_alone(pp, fresh):
    """NaN and infinite queries change their own rows only; the same call twice gives the same bits."""
    torch.manual_seed(7)
    length = [f + 300 for f in fresh]
    need = [-(-n // 16) for n in length]
    kc, vc = (torch.randn((sum(need), 16, 2, 64), device="cuda").to(torch.float16) for _ in range(2))
    table, at = np.zeros((4, 40)), 0
    for r, n in enumerate(need):
        table[r, :n] = np.arange(at, at + n)
        at += n
    q = torch.randn((sum(fresh), 8, 64), device="cuda").to(torch.float16)
    args = (_i32(table), _i32(np.concatenate([[0], np.cumsum(fresh)])), _i32(length), max(fresh))
    clean, again, out = (torch.empty_like(q) for _ in range(3))
    with pp.KVCache.like(kc) as kv:
        pp.pp_paged_attention(kv, q, kc, vc, *args, clean, 0.125)
        pp.pp_paged_attention(kv, q, kc, vc, *args, again, 0.125)
        bad = q.clone()
        bad[1, 3, 5] = float("nan")
        bad[2, 7] = float("inf")
        pp.pp_paged_attention(kv, bad, kc, vc, *args, out, 0.125)
        kv.sync()
    assert torch.equal(clean.view(torch.int16), again.view(torch.int16))
    hit = torch.zeros(out.shape[:2], dtype=torch.bool, device="cuda")
    hit[1, 3] = hit[2, 7] = True
    assert torch.equal(out[~hit], clean[~hit]) and out[hit].isnan().all()


def test_chunks_in_a_graph(pp):
    torch.manual_seed(8)
    kc, vc = (torch.randn((64, 16, 2, 128), device="cuda").to(torch.bfloat16) for _ in range(2))
    table = _i32(np.arange(64).reshape(2, 32))
    q_start, lens = _i32([0, 60, 200]), _i32([500, 300])
    q = torch.randn((200, 8, 128), device="cuda").to(torch.bfloat16)
    out = torch.empty_like(q)
    with pp.KVCache.like(kc) as kv:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            pp.pp_paged_attention(kv, q, kc, vc, table, q_start, lens, 140, out, 0.09)
        q_start.copy_(_i32([0, 100, 180]))
        lens.copy_(_i32([100, 512]))
        out.fill_(2)
        graph.replay()
        kv.sync()
    want, _, tol, _ = ref.attention(q[:180], kc, vc, table, [0, 100, 180], [100, 512], 0.09, 0)
    assert not ((out[:180].double() - want).abs() > tol).any() and (out[180:] == 2).all()


def test_block_tables_in_unaligned_buffers(pp):
    """Slot map and positions that start between 16-byte boundaries."""
    slots = torch.zeros(101, dtype=torch.int64, device="cuda")[1:]
    pos = torch.zeros(103, dtype=torch.int32, device="cuda")[3:]
    table = _i32(np.full((2, 8), -1))
    with pp.KVCache(20, 16, 1, 8) as kv:
        q, out = _i32([0] * 3), _i32([0])
        pp.pp_block_tables(kv, _i32([50, 37]), _i32([0, 0]), table, slots, pos, q, _i32(np.arange(20)[::-1].copy()),
                           _i32([2]), out)
        kv.sync()
    want = ref.block_tables([50, 37], [0, 0], None, None, np.full((2, 8), -1), np.arange(20)[::-1], 2, 16, 100)
    for got, exp in zip((table, slots, pos, q, out[0]), want):
        assert np.array_equal(got.cpu().numpy(), exp)


# few rows (new tokens x heads of a group) take the kernel of single tokens up to 32, the next one that of chunks
FEW = [([2, 1, 2], 4, 4), ([4, 3, 1, 0, 4], 8, 1), ([8, 5, 1], 8, 2), ([2, 2], 16, 1), ([3, 1], 14, 2), ([6, 2], 5, 1),
       ([32, 7, 0, 31], 2, 2), ([33, 1], 2, 2), ([5, 2], 14, 2), ([1, 1], 33, 1)]


@pytest.mark.parametrize("fresh,heads,kv_heads", FEW)
@pytest.mark.parametrize("dim,dtype,block,order", [(128, torch.bfloat16, 16, "token"), (64, torch.float16, 8, "head"),
                                                   (80, torch.float16, 64, "token")])
def test_few_rows(pp, fresh, heads, kv_heads, dim, dtype, block, order):
    cached = [0, 901, 127, 128, 3000][:len(fresh)]
    _attention_case(pp, fresh, cached, heads, kv_heads, dim, dtype, block=block, order=order)


@pytest.mark.parametrize("window", [1, 2, 3, 17, 128, 129, 700])
@pytest.mark.parametrize("fresh,heads,kv_heads", [([4, 1, 3], 8, 2), ([4, 2], 8, 1), ([32, 20], 1, 1)])
def test_few_rows_window(pp, fresh, heads, kv_heads, window):
    _attention_case(pp, fresh, [1000, 255, 0][:len(fresh)], heads, kv_heads, 128, window=window)


def test_few_rows_that_see_nothing(pp):
    """The first queries stand before the first key, the last request has no token at all."""
    out = _attention_case(pp, [4, 8, 3], [-2, -7, -3], 8, 2, 64)
    assert int((out[:2] != 0).sum()) == 0 and int((out[4:11] != 0).sum()) == 0


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("fresh,row", [([2], 202), ([4], 203), ([4], 190), ([8], 204), ([10], 100)])
@pytest.mark.parametrize("window", [0, 12])
def test_few_rows_values_out_of_range(pp, bad, fresh, row, window):
    test_values_out_of_range_stay_with_those_who_see_them(pp, bad, fresh, row, window)


@pytest.mark.parametrize("fresh,row", [([2], 202), ([10], 207), ([7], 120)])
def test_few_rows_nan_key(pp, fresh, row):
    test_a_nan_key_stays_with_those_who_see_it(pp, fresh, row)


@pytest.mark.parametrize("fresh,cached,heads,kv_heads,dim", [
    ([100], [20_000], 8, 1, 128), ([100], [20_000], 8, 2, 64), ([65, 65, 65], [9000, 11_000, 300], 4, 1, 128),
    ([300, 1, 33], [7000, 20_000, 5], 8, 2, 128), ([33], [30_000], 1, 1, 72)])
def test_many_pieces(pp, fresh, cached, heads, kv_heads, dim):
    """Items that many CTAs compute, joined in shares."""
    _attention_case(pp, fresh, cached, heads, kv_heads, dim)


@pytest.mark.parametrize("dim", [64, 128])
def test_many_pieces_again_and_again(pp, dim):
    """Calls of one handle by turns: the same bits each time, whoever joins, and nothing left behind."""
    torch.manual_seed(9)
    kc, vc = (torch.randn((1300, 16, 2, dim), device="cuda").to(torch.bfloat16) for _ in range(2))
    calls = []
    for fresh, length in ([[40], [20_000]], [[30, 50], [5000, 9000]], [[4], [20_000]], [[90, 3, 200], [300, 6000, 8000]]):
        n = sum(fresh)
        table = torch.arange(1300, dtype=torch.int32, device="cuda").repeat(len(fresh), 1)
        q = torch.randn((n, 8, dim), device="cuda").to(torch.bfloat16)
        calls.append((q, table, _i32(np.concatenate([[0], np.cumsum(fresh)])), _i32(length), max(fresh)))
    first = {}
    with pp.KVCache.like(kc) as kv:
        for turn in range(25):
            for i, (q, *args) in enumerate(calls):
                out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
                pp.pp_paged_attention(kv, q, kc, vc, *args, out, 0.1, lse=lse)
                want = first.setdefault(i, (out, lse))
                assert torch.equal(out.view(torch.int16), want[0].view(torch.int16)) and torch.equal(lse, want[1])
        kv.sync()
    for i, (q, table, q_start, length, _) in enumerate(calls):
        want, _, tol, _ = ref.attention(q, kc, vc, table, q_start.tolist(), length.tolist(), 0.1, 0)
        assert not ((first[i][0].double() - want).abs() > tol).any()


def test_refuses_too_many_heads(pp):
    kc, vc = (torch.zeros((1, 16, 1, 8), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q = torch.zeros((1, (1 << 20) + 1, 8), dtype=torch.bfloat16, device="cuda")
    with pp.KVCache.like(kc) as kv:
        with pytest.raises(pp.PPError, match="at most 2\\^20"):
            pp.pp_paged_attention(kv, q, kc, vc, _i32([[0]]), _i32([0, 1]), _i32([1]), 1, torch.empty_like(q), 0.1)


def test_two_handles_on_two_streams(pp):
    """Calls whose joins many CTAs share, at the same time: each has its own scratch, and neither waits for the other."""
    torch.manual_seed(10)
    kc, vc = (torch.randn((700, 16, 2, 128), device="cuda").to(torch.bfloat16) for _ in range(2))
    table = torch.arange(700, dtype=torch.int32, device="cuda")[None]
    calls = []
    for fresh, length in ((50, 11_000), (300, 10_000), (2, 11_200)):
        q = torch.randn((fresh, 8, 128), device="cuda").to(torch.bfloat16)
        calls.append((q, table, _i32([0, fresh]), _i32([length]), fresh))
    outs = [[], []]
    torch.cuda.synchronize()
    with pp.KVCache.like(kc) as one, pp.KVCache.like(kc) as two:
        streams = torch.cuda.Stream(), torch.cuda.Stream()
        for turn in range(10):
            for kv, stream, out in zip((one, two), streams, outs):
                with torch.cuda.stream(stream):
                    for q, *args in calls:
                        out.append(torch.empty_like(q))
                        pp.pp_paged_attention(kv, q, kc, vc, table, *args[1:], out[-1], 0.1)
        torch.cuda.synchronize()
        one.sync()
        two.sync()
    for i, (q, _, q_start, length, _) in enumerate(calls):
        want, _, tol, _ = ref.attention(q, kc, vc, table, q_start.tolist(), length.tolist(), 0.1, 0)
        assert not ((outs[0][i].double() - want).abs() > tol).any()
        for out in outs:
            for turn in range(10):
                assert torch.equal(out[3 * turn + i].view(torch.int16), outs[0][i].view(torch.int16))
