"""pp_kv_write8 against its plain form (kv8_reference.py): codes and exponents are equal."""
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


class _Cache:
    """K and V caches of 8-bit numbers, any codes and exponents at first, beside what they should hold."""

    def __init__(self, blocks, block, heads, dim, dtype, order="token", seed=0):
        self.rng = np.random.default_rng(seed)
        self.block, self.dtype = block, dtype
        shape = (blocks, block, heads, dim) if order == "token" else (blocks, heads, block, dim)
        self.code, self.exp, self.want = [], [], []
        for _ in range(2):
            raw = torch.tensor(self.rng.integers(0, 256, size=shape), dtype=torch.uint8, device="cuda")
            code = raw.view(torch.float8_e4m3fn)
            self.code.append(code if order == "token" else code.transpose(1, 2))
            self.exp.append(torch.tensor(self.rng.integers(-12, 4, size=(blocks, heads)), dtype=torch.int8, device="cuda"))
            self.want.append((ref.values(self.code[-1]), self.exp[-1].cpu().numpy()))

    def write(self, pp, kv, k, v, slot, **kw):
        slot_t = torch.as_tensor(np.asarray(slot, np.int64), device="cuda")
        pp.pp_kv_write8(kv, k, v, slot_t, self.code[0], self.exp[0], self.code[1], self.exp[1], **kw)
        self.expect(k, v, slot)

    def expect(self, k, v, slot):
        self.want = [ref.write8(x.double().cpu().numpy(), slot, *w, self.block) for x, w in zip((k, v), self.want)]

    def check(self):
        for name, code, exp, (wc, we) in zip("kv", self.code, self.exp, self.want):
            assert np.array_equal(exp.cpu().numpy(), we), name
            got = ref.values(code)
            same = (got == wc) | (np.isnan(got) & np.isnan(wc))
            assert same.all(), f"{name}: {int((~same).sum())} codes differ, first at {np.argwhere(~same)[0]}"


def _rows(tokens, heads, dim, dtype, spread=1.0):
    """Rows of a projection's output, of sizes over some binades."""
    x = torch.randn((tokens, heads + 1, dim), device="cuda") * torch.exp2(torch.randn((tokens, heads + 1, 1), device="cuda") * spread)
    return x.to(dtype)[:, 1:]


def _runs(rng, blocks, block, count, whole=0.3):
    """Slots of `count` requests, each from a place in its block on over some blocks; tokens left out among them."""
    ids, at, slot = rng.permutation(blocks), 0, []
    for _ in range(count):
        first = 0 if rng.random() < whole else int(rng.integers(0, block))
        n = int(rng.integers(1, 3 * block))
        if at + (first + n - 1) // block + 1 > blocks:
            break
        place = first + np.arange(n)
        slot += (ids[at + place // block] * block + place % block).tolist()
        at += (first + n - 1) // block + 1
    slot = np.array(slot)
    slot[rng.random(len(slot)) < 0.1] = -1
    return slot


@pytest.mark.parametrize("block", [8, 16, 32, 64, 128, 256, 512])
@pytest.mark.parametrize("order", ["token", "head"])
@pytest.mark.parametrize("heads,dim,dtype", [(1, 16, BF), (3, 80, HF), (4, 128, BF)])
def test_runs(pp, block, order, heads, dim, dtype):
    """Requests' new rows, in several calls over the same blocks."""
    torch.manual_seed(block)
    c = _Cache(12, block, heads, dim, dtype, order, seed=block + dim)
    with pp.KVCache.like(c.code[0], dtype=dtype) as kv:
        for _ in range(3):
            slot = _runs(c.rng, 12, block, 6)
            c.write(pp, kv, _rows(len(slot), heads, dim, dtype, 3.0), _rows(len(slot), heads, dim, dtype, 3.0), slot)
            kv.sync()
            c.check()


@pytest.mark.parametrize("tokens", [1, 2, 31, 32, 33, 304, 305, 1000, 5000])
@pytest.mark.parametrize("heads", [1, 2, 9])
def test_single_rows(pp, tokens, heads):
    """A decode step: a row in a block of each request, at any place."""
    torch.manual_seed(tokens)
    c = _Cache(tokens + 2, 16, heads, 64, BF, seed=tokens)
    slot = c.rng.permutation(tokens + 2)[:tokens] * 16 + c.rng.integers(0, 16, size=tokens)
    with pp.KVCache.like(c.code[0]) as kv:
        c.write(pp, kv, _rows(tokens, heads, 64, BF, 2.0), _rows(tokens, heads, 64, BF, 2.0), slot)
        kv.sync()
    c.check()


@pytest.mark.parametrize("block,tokens,dim", [(8, 9000, 64), (16, 40_000, 128), (32, 20_000, 16), (64, 20_000, 128),
                                              (128, 15_000, 80), (256, 15_000, 32), (512, 40_000, 128)])
def test_many_tokens(pp, block, tokens, dim):
    """More tokens than a CTA looks at together; runs of one, few and many rows next to one another."""
    torch.manual_seed(block)
    rng = np.random.default_rng(block)
    slot, at = [], 0
    while len(slot) < tokens:
        first = 0 if rng.random() < 0.3 else int(rng.integers(0, block))
        n = int(rng.choice([1, 1, 1, 2, 3, 17, 40, 3 * block]))
        place = first + np.arange(n)
        slot += ((at + place // block) * block + place % block).tolist()
        at += (first + n - 1) // block + 1
    slot = np.array(slot[:tokens])
    slot[rng.random(tokens) < 0.02] = -1
    c = _Cache(at, block, 1, dim, BF, seed=block)
    with pp.KVCache.like(c.code[0]) as kv:
        c.write(pp, kv, _rows(tokens, 1, dim, BF, 2.0), _rows(tokens, 1, dim, BF, 2.0), slot)
        kv.sync()
    c.check()


def test_a_block_that_grows_token_by_token(pp):
    """The scale only grows, until the block is begun anew."""
    c = _Cache(2, 16, 2, 32, HF, seed=5)
    with pp.KVCache.like(c.code[0], dtype=HF) as kv:
        for step in range(36):
            x = torch.randn((1, 2, 32), device="cuda").mul_(2.0 ** ((step * 7) % 19 - 9)).to(HF)
            c.write(pp, kv, x, -x, [16 + step % 16])
            c.check()
        kv.sync()


@pytest.mark.parametrize("gap", [1, 31])
@pytest.mark.parametrize("first", [0, 3, 30, 31])
def test_tokens_left_out_within_a_block(pp, gap, first):
    """Rows of one block with tokens left out between them count together, wherever a CTA's tokens begin."""
    c = _Cache(5, 16, 1, 16, BF, seed=gap)
    slot = [-1] * first
    for i in range(5):
        slot += [48 + 2 + i] + [-1] * gap
    slot += [16, 17, -9, 18] + [-1] * 40
    slot += [64 + 1] * 1 + [-1] * 700
    with pp.KVCache.like(c.code[0]) as kv:
        c.write(pp, kv, _rows(len(slot), 1, 16, BF, 3.0), _rows(len(slot), 1, 16, BF, 3.0), slot)
        kv.sync()
    c.check()


def test_any_order_within_a_block(pp):
    c = _Cache(9, 64, 2, 48, HF, seed=2)
    slot = np.concatenate([b * 64 + c.rng.permutation(64)[:n] for b, n in ((7, 64), (2, 1), (0, 33), (3, 64))])
    with pp.KVCache.like(c.code[0], dtype=HF) as kv:
        c.write(pp, kv, _rows(len(slot), 2, 48, HF, 2.0), _rows(len(slot), 2, 48, HF, 2.0), slot)
        kv.sync()
    c.check()


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("begun", [False, True])
def test_every_number(pp, dtype, begun):
    """All numbers of the type, in blocks of like sizes and of all sizes: borders of scales, ties, the smallest and
    largest, infinities, NaN, zeros of both signs."""
    raw = torch.arange(-(1 << 15), 1 << 15, dtype=torch.int32, device="cuda").to(torch.int16).view(dtype)
    mixed = raw[torch.randperm(1 << 16, generator=torch.Generator().manual_seed(1)).cuda()]
    c = _Cache(70, 16, 2, 32, dtype, seed=9)
    with pp.KVCache.like(c.code[0], dtype=dtype) as kv:
        k, v = raw.view(-1, 2, 32), mixed.view(-1, 2, 32)
        slot = np.arange(1024) if begun else (np.arange(1024) // 15 * 16 + 1 + np.arange(1024) % 15)
        c.write(pp, kv, k, v, slot)
        kv.sync()
    c.check()


@pytest.mark.parametrize("value,exponent", [(0.0, -40), (448.0, 0), (449.0, 1), (448 * 2.0 ** -40, -40), (2.0 ** -60, -40),
                                            (448 * 2.0 ** 40, 40), (3e38, 40), (1.0, -8), (1.75, -8), (1.7578125, -7)])
def test_exponents(pp, value, exponent):
    c = _Cache(1, 8, 1, 16, BF, seed=1)
    x = torch.zeros((1, 1, 16), dtype=BF, device="cuda")
    x[0, 0, 5] = -value
    assert abs(float(x[0, 0, 5])) == pytest.approx(value, rel=2 ** -8)
    with pp.KVCache.like(c.code[0]) as kv:
        c.write(pp, kv, x, x, [0])
        kv.sync()
    c.check()
    want = next((e for e in range(-40, 40) if abs(float(x[0, 0, 5])) <= 448 * 2.0 ** e), 40)
    assert int(c.exp[0][0, 0]) == want and (want == exponent or value in (449.0, 1.7578125))


def test_nothing_finite(pp):
    """Rows of infinities and NaN alone do not move the scale."""
    c = _Cache(2, 8, 1, 16, HF, seed=4)
    x = torch.full((2, 1, 16), math.inf, dtype=HF, device="cuda")
    x[:, :, ::2] = math.nan
    with pp.KVCache.like(c.code[0], dtype=HF) as kv:
        c.write(pp, kv, x, -x, [0, 13])
        kv.sync()
    c.check()
    assert int(c.exp[0][0, 0]) == -40 and np.isnan(ref.values(c.code[0])[0, 0]).all()


def test_exponents_outside_the_range_are_read_as_its_ends(pp):
    c = _Cache(3, 8, 1, 16, BF, seed=6)
    for i in range(2):
        c.exp[i][:] = torch.tensor([[-128], [127], [41]], dtype=torch.int8, device="cuda")
    c.want = [(w[0], e.cpu().numpy()) for w, e in zip(c.want, c.exp)]
    with pp.KVCache.like(c.code[0]) as kv:
        x = _rows(3, 1, 16, BF)
        c.write(pp, kv, x, x, [1, 9, 17])
        kv.sync()
    c.check()


def test_bounds(pp):
    c = _Cache(2, 8, 1, 16, BF, seed=7)
    x = _rows(5, 1, 16, BF)
    with pp.KVCache.like(c.code[0]) as kv:
        c.write(pp, kv, x, x, [16, 3, 1 << 40, 4, -1])
        with pytest.raises(pp.PPError, match="PP_EBOUNDS"):
            kv.sync()
        kv.sync()
    c.check()


def test_no_tokens(pp):
    c = _Cache(2, 8, 1, 16, BF)
    with pp.KVCache.like(c.code[0]) as kv:
        empty = torch.empty((0, 1, 16), dtype=BF, device="cuda")
        c.write(pp, kv, empty, empty, [])
        kv.sync()
    c.check()


def test_refusals(pp):
    c = _Cache(2, 16, 2, 64, BF)
    rows = torch.randn((3, 2, 72), device="cuda").to(BF)
    slot = torch.tensor([0, 1, 2], device="cuda")
    good = dict(k=rows[..., :64], v=rows[..., 8:], slot_map=slot, k_cache=c.code[0], k_exp=c.exp[0], v_cache=c.code[1], v_exp=c.exp[1])
    wide = torch.zeros((2, 16, 2, 64), dtype=BF, device="cuda")
    with pp.KVCache.like(c.code[0]) as kv:
        for bad in (dict(k=rows[..., 4:68]), dict(v=torch.zeros((3, 2, 68), dtype=BF, device="cuda")[..., :64]),
                    dict(v_cache=c.code[0]), dict(v_exp=c.exp[0])):
            with pytest.raises(pp.PPError, match="PP_EINVAL"):
                pp.pp_kv_write8(kv, **{**good, **bad})
        with pytest.raises(ValueError):
            pp.pp_kv_write(kv, good["k"], good["v"], slot, wide, wide)
        assert pp._lib.pp_kv_write(kv.handle, 3, wide.data_ptr(), 128, 64, wide.data_ptr(), 128, 64, slot.data_ptr(),
                                   wide.data_ptr(), wide.data_ptr(), None) == pp.PP_EINVAL
        kv.sync()
    c.check()
    with pp.KVCache.like(wide) as kv:
        assert pp._lib.pp_kv_write8(kv.handle, 3, wide.data_ptr(), 128, 64, wide.data_ptr(), 128, 64, slot.data_ptr(),
                                    wide.data_ptr(), c.exp[0].data_ptr(), wide.data_ptr(), c.exp[1].data_ptr(), None) == pp.PP_EINVAL
        with pytest.raises(ValueError, match="eight_bit"):
            pp.pp_kv_write8(kv, **good)
    with pytest.raises(ValueError, match="rows of a"):
        pp.KVCache.like(wide, dtype=HF)


def test_graph_and_streams(pp):
    c = _Cache(40, 16, 2, 128, BF, seed=3)
    k, v = (torch.randn((30, 2, 128), device="cuda").to(BF) for _ in range(2))
    place = np.arange(30) * 16 + 3
    slot = torch.tensor(place, device="cuda")
    with pp.KVCache.like(c.code[0]) as kv:
        call = lambda **kw: pp.pp_kv_write8(kv, k, v, slot, c.code[0], c.exp[0], c.code[1], c.exp[1], **kw)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        call(stream=side)
        kv.sync(side)
        c.expect(k, v, place)
        c.check()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        for step in range(3):
            k.copy_(torch.randn_like(k) * 4 ** step)
            v.copy_(torch.randn_like(v) * 4 ** step)
            slot += 1
            place += 1
            graph.replay()
            kv.sync()
            c.expect(k, v, place)
            c.check()
