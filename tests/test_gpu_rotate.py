"""pp_kv_rotate against its 64-bit form (kv8_reference.py), at the layouts, sizes and positions
where it can go wrong, and its refusals."""
import math

import numpy as np
import pytest

from tests import kv8_reference as ref

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


def _rows(tokens, heads, dim, dtype, gen=None):
    """Rows between others, as in a projection's output, whose neighbours are NaN."""
    t = torch.full((tokens, heads + 2, dim + 8), math.nan, dtype=dtype, device="cuda")
    t[:, 1:1 + heads, :dim] = torch.randn((tokens, heads, dim), device="cuda").mul_(3).to(dtype)
    return t[:, 1:1 + heads, :dim]


def _positions(tokens, longest, seed=0):
    rng = np.random.default_rng(seed)
    p = rng.integers(-3, longest, size=tokens)
    p[:4] = [longest - 1, 0, 1, -1][:min(4, tokens)]
    return torch.tensor(p, dtype=torch.int32, device="cuda")


def _check(got, want, what):
    out, tol = want
    err = (got.double() - out).abs()
    assert not (err > tol).any() and not err.isnan().any(), \
        f"{what}: {int((~(err <= tol)).sum())} of {err.numel()} out of bound, worst {float((err / tol.clamp(min=1e-30)).max())}"


def _case(pp, tokens, heads, kv_heads, dim, rotated, interleaved, dtype, norm, to="rows", longest=100_000, block=16,
          in_place=False, amplitude=1.0, eps=1e-5, **scaling):
    torch.manual_seed(tokens + dim)
    q = _rows(tokens, heads, dim, dtype) if heads else None
    k, v = _rows(tokens, kv_heads, dim, dtype), _rows(tokens, kv_heads, dim, dtype)
    weight = [(torch.randn(dim, device="cuda") * 0.5 + 1).to(dtype) if x else None for x in norm]
    position = _positions(tokens, longest)
    rotary = pp.Rotary(rotated, amplitude=amplitude, interleaved=interleaved, **scaling)
    args = (position, rotary.frequencies, rotated, interleaved, amplitude)
    wq = ref.rotate(q, weight[0], eps, *args) if heads else None
    wk = ref.rotate(k, weight[1], eps, *args)
    blocks = tokens // block + 2
    kc, vc = (torch.full((blocks, block, kv_heads, dim), 7.0, dtype=dtype, device="cuda") for _ in range(2))
    ec, ev = kc.double(), vc.clone()
    slot = torch.randperm(blocks * block, device="cuda")[:tokens]
    slot[::5] = -1 - slot[::5]
    keep = slot >= 0
    q_out = None if not heads else q if in_place else torch.full_like(q, 5.0)
    k_out = k if in_place else torch.full((tokens, kv_heads, dim), 5.0, dtype=dtype, device="cuda")
    more = {}
    if to != "rows":
        more = dict(v=v, slot_map=slot, k_cache=kc, v_cache=vc)
        if to == "cache":
            k_out = None
    with pp.KVCache.like(kc) as kv:
        pp.pp_kv_rotate(kv, rotary, q, k, position, q_out, k_out=k_out, q_weight=weight[0], k_weight=weight[1], eps=eps, **more)
        kv.sync()
    if heads:
        _check(q_out, wq, "q")
    if k_out is not None:
        _check(k_out, wk, "k")
    if to != "rows":
        tol = torch.zeros_like(ec)
        ec[slot[keep] // block, slot[keep] % block] = wk[0][keep]
        tol[slot[keep] // block, slot[keep] % block] = wk[1][keep]
        ev[slot[keep] // block, slot[keep] % block] = v[keep]
        _check(kc, (ec, tol), "k_cache")
        assert torch.equal(vc, ev)
    else:
        assert (kc == 7).all() and (vc == 7).all()


BF, HF = torch.bfloat16, torch.float16


@pytest.mark.parametrize("dim,rotated", [(8, 8), (8, 2), (8, 6), (16, 16), (16, 4), (40, 40), (40, 16), (40, 10), (64, 64),
                                         (64, 32), (72, 18), (80, 80), (80, 20), (80, 32), (96, 48), (128, 128),
                                         (128, 64), (128, 2), (128, 126), (128, 0)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("norm", [(False, False), (True, True)])
def test_layouts(pp, dim, rotated, interleaved, norm):
    _case(pp, 37, 6, 2, dim, rotated, interleaved, BF if dim % 16 else HF, norm)


@pytest.mark.parametrize("heads,kv_heads", [(0, 1), (1, 1), (7, 1), (3, 3), (28, 4), (40, 8), (130, 65)])
@pytest.mark.parametrize("tokens", [1, 5, 333])
@pytest.mark.parametrize("to", ["rows", "cache", "both"])
def test_heads_and_targets(pp, heads, kv_heads, tokens, to):
    _case(pp, tokens, heads, kv_heads, 128, 128, False, BF, (True, True), to)
    _case(pp, tokens, heads, kv_heads, 80, 40, True, HF, (False, False), to, block=8)


@pytest.mark.parametrize("norm", [(True, False), (False, True)])
@pytest.mark.parametrize("dim,rotated", [(128, 128), (80, 20)])
@pytest.mark.parametrize("tokens", [2, 200])
def test_one_of_the_norms(pp, norm, dim, rotated, tokens):
    """Lanes of a warp have rows of q and of k at once."""
    _case(pp, tokens, 5, 3, dim, rotated, False, BF, norm, "both")


@pytest.mark.parametrize("dim,rotated,interleaved", [(128, 128, False), (128, 64, True), (80, 20, False), (40, 10, False)])
@pytest.mark.parametrize("tokens", [3, 700])
def test_in_place(pp, dim, rotated, interleaved, tokens):
    _case(pp, tokens, 9, 3, dim, rotated, interleaved, BF, (True, True), in_place=True)


@pytest.mark.parametrize("longest", [1 << 20, 1 << 31])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_far_positions(pp, longest, dtype):
    """The first pair turns by a radian a token: a 32-bit product would be off by whole turns."""
    _case(pp, 300, 2, 1, 64, 64, False, dtype, (False, False), longest=longest)
    _case(pp, 300, 2, 1, 64, 64, True, dtype, (False, False), longest=longest, factor=4.0, original=8192, amplitude=1.14)


def test_given_frequencies(pp):
    f = np.array([3.5, -1.0, 0.0, 1e-3, 100.0, 2 * math.pi, 1e-9, 0.25])
    _case(pp, 50, 3, 1, 16, 16, False, HF, (False, False), longest=5000, frequencies=f)


@pytest.mark.parametrize("dtype", [BF, HF])
def test_norm_of_zero_and_large_rows(pp, dtype):
    """A row of zeros stays one (eps); large rows overflow no sum."""
    dim, big = 64, 60000.0 if dtype == HF else 1e18
    q = torch.zeros((3, 1, dim), dtype=dtype, device="cuda")
    q[1], q[2] = big, 1e-3
    w = torch.ones(dim, dtype=dtype, device="cuda")
    out, ko = torch.empty_like(q), torch.empty_like(q)
    with pp.KVCache(1, 16, 1, dim, dtype) as kv:
        pp.pp_kv_rotate(kv, None, q, q, torch.zeros(3, dtype=torch.int32, device="cuda"), out, k_out=ko, q_weight=w, eps=1e-6)
        kv.sync()
    want = q.double() / torch.sqrt(q.double().square().mean(-1, keepdim=True) + 1e-6)
    assert ((out.double() - want).abs() <= 1.01 * ref.UNIT[dtype] * want.abs()).all()
    assert torch.equal(ko, q)                               # neither normed nor rotated


def test_bits_of_rows_left_alone(pp):
    """Without norm and rotation rows keep their bits, infinities, NaN and -0 among them; so do elements that do not turn."""
    raw = torch.arange(-(1 << 15), 1 << 15, dtype=torch.int32, device="cuda").to(torch.int16)
    for dtype in (BF, HF):
        rows = raw.view(dtype).view(-1, 4, 128)
        finite = torch.nan_to_num(rows, 0.0, 1.0, 1.0)
        position = torch.arange(len(rows), dtype=torch.int32, device="cuda")
        with pp.KVCache(1, 16, 4, 128, dtype) as kv:
            q_out, k_out = torch.zeros_like(rows), torch.zeros_like(rows)
            pp.pp_kv_rotate(kv, None, rows, rows, position, q_out, k_out=k_out)
            assert torch.equal(q_out.view(torch.int16)[~rows.isnan()], rows.view(torch.int16)[~rows.isnan()])
            assert q_out[rows.isnan()].isnan().all() and torch.equal(q_out.view(torch.int16), k_out.view(torch.int16))
            for rotated, inter in ((32, False), (32, True), (20, False)):
                mixed = torch.cat((finite[..., :rotated], rows[..., rotated:]), -1)
                pp.pp_kv_rotate(kv, pp.Rotary(rotated, interleaved=inter), mixed, mixed, position, q_out, k_out=k_out)
                tail = rows[..., rotated:]
                keep = ~tail.isnan()
                assert torch.equal(q_out[..., rotated:].contiguous().view(torch.int16)[keep], tail.contiguous().view(torch.int16)[keep])
                assert not q_out[..., :rotated].isnan().any()
            kv.sync()


def test_no_tokens(pp):
    with pp.KVCache(1, 16, 2, 64) as kv:
        empty = torch.empty((0, 2, 64), dtype=BF, device="cuda")
        pp.pp_kv_rotate(kv, pp.Rotary(64), empty, empty, torch.empty(0, dtype=torch.int32, device="cuda"), empty, k_out=empty)
        kv.sync()


def test_slots_out_of_range(pp):
    kc, vc = (torch.zeros((2, 8, 1, 16), dtype=BF, device="cuda") for _ in range(2))
    rows = torch.ones((4, 1, 16), dtype=BF, device="cuda")
    with pp.KVCache.like(kc) as kv:
        pp.pp_kv_rotate(kv, None, None, rows, torch.zeros(4, dtype=torch.int32, device="cuda"), None, v=rows,
                        slot_map=torch.tensor([16, 3, 1 << 40, -5], device="cuda"), k_cache=kc, v_cache=vc)
        with pytest.raises(pp.PPError, match="PP_EBOUNDS"):
            kv.sync()
        kv.sync()
    assert int(kc.sum()) == 16 and int(kc[0, 3].sum()) == 16 and int(vc.sum()) == 16


def test_8_bit_handles_rotate_to_rows_only(pp):
    cache = torch.zeros((2, 16, 2, 64), dtype=torch.float8_e4m3fn, device="cuda")
    rows = torch.randn((5, 2, 64), device="cuda").to(HF)
    position = torch.arange(5, dtype=torch.int32, device="cuda")
    slot = torch.arange(5, device="cuda")
    with pp.KVCache.like(cache, dtype=HF) as kv:
        out, k_out = torch.empty_like(rows), torch.empty_like(rows)
        rotary = pp.Rotary(64)
        pp.pp_kv_rotate(kv, rotary, rows, rows, position, out, k_out=k_out)
        kv.sync()
        _check(out, ref.rotate(rows, None, 0, position, rotary.frequencies, 64, False, 1.0), "q")
        assert torch.equal(out, k_out)
        with pytest.raises(pp.PPError, match="pp_kv_write8"):
            pp.pp_kv_rotate(kv, rotary, rows, rows, position, out, k_out=k_out, v=rows, slot_map=slot, k_cache=cache, v_cache=cache)


def test_refusals(pp):
    kc, vc = (torch.full((2, 16, 2, 64), 3.0, dtype=BF, device="cuda") for _ in range(2))
    base = torch.full((1 << 14,), 3.0, dtype=BF, device="cuda")
    rows = base[:5 * 128].view(5, 2, 64)
    out, ko = base[1024:1664].view(5, 2, 64), base[2048:2688].view(5, 2, 64)
    position = torch.arange(5, dtype=torch.int32, device="cuda")
    slot = torch.arange(5, device="cuda")
    r = pp.Rotary(64)
    good = dict(rotary=r, q=rows, k=rows, position=position, q_out=out, k_out=ko)
    caches = dict(v=rows, slot_map=slot, k_cache=kc, v_cache=vc)
    at = lambda first, *st: base.as_strided((5, 2, 64), (*st, 1), first)
    bad = [
        dict(k_out=None), dict(eps=-1.0), dict(eps=math.nan), dict(eps=math.inf),
        *[{k: v for k, v in caches.items() if k != name} for name in caches],
        dict(q=at(4, 128, 64)), dict(q=at(0, 132, 64)), dict(q_out=at(1, 128, 64)), dict(k=at(2, 128, 64)), dict(k_out=at(4, 128, 64)),
        dict(q_out=at(1024, 64, 64)), dict(k_out=at(1024, 64, 128 + 64)), dict(k_out=at(1024, 128, 8)),
        dict(q_out=at(0, 256, 64)), dict(k_out=at(0, 128, 5 * 128)),     # over the inputs, other strides
        dict(q_weight=base[1:65]),
    ]
    with pp.KVCache.like(kc) as kv:
        amplitude = pp.Rotary(64, amplitude=math.nan)
        for change in bad + [dict(rotary=amplitude)]:
            with pytest.raises(pp.PPError, match="PP_EINVAL"):
                pp.pp_kv_rotate(kv, **{**good, **change})
        kv.sync()
        assert (base == 3).all() and (kc == 3).all() and (vc == 3).all()
        pp.pp_kv_rotate(kv, **good)
        kv.sync()


def test_graph_and_streams(pp):
    """Captured and replayed with new inputs in the same buffers; launched on a stream of its own."""
    torch.manual_seed(3)
    q, k = (torch.randn((40, h, 128), device="cuda").to(BF) for h in (8, 2))
    v = torch.randn_like(k)
    kc, vc = (torch.zeros((8, 16, 2, 128), dtype=BF, device="cuda") for _ in range(2))
    position, slot = torch.arange(40, dtype=torch.int32, device="cuda"), torch.arange(40, device="cuda")
    q_out, rotary = torch.empty_like(q), pp.Rotary(128)
    with pp.KVCache.like(kc) as kv:
        call = lambda **kw: pp.pp_kv_rotate(kv, rotary, q, k, position, q_out, v=v, slot_map=slot, k_cache=kc, v_cache=vc, **kw)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        call(stream=side)
        kv.sync(side)
        want = ref.rotate(q, None, 0, position, rotary.frequencies, 128, False, 1.0)
        _check(q_out, want, "q")
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        for step in range(3):
            q.copy_(torch.randn_like(q))
            k.copy_(torch.randn_like(k))
            position += 1000
            graph.replay()
            kv.sync()
            _check(q_out, ref.rotate(q, None, 0, position, rotary.frequencies, 128, False, 1.0), "q")
            _check(kc.view(-1, 2, 128)[:40], ref.rotate(k, None, 0, position, rotary.frequencies, 128, False, 1.0), "k")
            assert torch.equal(vc.view(-1, 2, 128)[:40], v)
