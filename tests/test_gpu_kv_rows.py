"""A row's result depends on what the row sees and on nothing else: not on the rows that
share a warp, a tile or a K/V head with it.  Sizes at which every CTA has several tiles of
an item, so that what is done once an item and what is done for each tile both run."""
import math

import numpy as np
import pytest

from tests.kv_tiles import chunk_tiles

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


# fresh tokens after cached ones, K/V heads, query heads, width, type, window
SIZES = [(2048, 2048, 8, 8, 64, torch.float16, 0), (2048, 2048, 8, 8, 128, torch.bfloat16, 0),
         (900, 3000, 6, 18, 128, torch.float16, 0), (2048, 2048, 24, 24, 64, torch.bfloat16, 900)]


class _Call:
    """One request over a cache in block order."""

    def __init__(self, pp, fresh, cached, kv_heads, heads, dim, dtype, window):
        sms = torch.cuda.get_device_properties(0).multi_processor_count
        assert chunk_tiles([fresh], [cached], heads // kv_heads, kv_heads, window) >= 8 * sms
        torch.manual_seed(11)
        self.pp, self.window, self.fresh, self.n = pp, window, fresh, fresh + cached
        blocks = -(-self.n // 16)
        self.kc, self.vc = (torch.randn((blocks, 16, kv_heads, dim), device="cuda").to(dtype) for _ in range(2))
        self.q = (1.5 * torch.randn((fresh, heads, dim), device="cuda")).to(dtype)
        self.table = torch.arange(blocks, dtype=torch.int32, device="cuda")[None]
        self.scale = dim ** -0.5

    def __call__(self, q=None):
        out = torch.empty_like(self.q)
        lse = torch.empty(self.q.shape[:2], device="cuda")
        with self.pp.KVCache.like(self.kc) as kv:
            self.pp.pp_paged_attention(kv, self.q if q is None else q, self.kc, self.vc, self.table, _i32([0, self.fresh]),
                                       _i32([self.n]), self.fresh, out, self.scale, window=self.window, lse=lse)
            kv.sync()
        return out, lse

    def sees(self, row):
        pos = torch.arange(self.n - self.fresh, self.n, device="cuda")
        return (pos >= row) & ((pos - row < self.window) if self.window else True)


@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("at", [333, 715])
@pytest.mark.parametrize("value", ["nan", "inf", "loud"])
def test_a_later_key_leaves_earlier_rows_alone(pp, size, at, value):
    """Rows before the key's share a warp with rows after it."""
    call = _Call(pp, *size)
    clean, clean_lse = call()
    row = call.n - call.fresh + at
    if value == "loud":
        call.kc[row // 16, row % 16] *= 30
    else:
        call.kc[row // 16, row % 16, :, 5] = float(value)
    out, lse = call()
    hidden = ~call.sees(row)
    assert int(hidden.sum()) >= at
    assert torch.equal(out[hidden], clean[hidden]) and torch.equal(lse[hidden], clean_lse[hidden])
    assert not clean.isnan().any()
    if value == "nan":
        assert out[~hidden].isnan().all()


@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("value", ["nan", "inf", "loud"])
def test_a_query_leaves_its_neighbours_alone(pp, size, value):
    call = _Call(pp, *size)
    clean, clean_lse = call()
    q = call.q.clone()
    hit = torch.zeros(q.shape[:2], dtype=torch.bool, device="cuda")
    for token, head in ((1, 0), (333, 2), (334, 3), (715, 5)):
        hit[token, head] = True
        if value == "loud":
            q[token, head] *= 30
        else:
            q[token, head, 5] = float(value)
    out, lse = call(q)
    assert torch.equal(out[~hit], clean[~hit]) and torch.equal(lse[~hit], clean_lse[~hit])
    assert not clean.isnan().any()
    if value == "nan":
        assert out[hit].isnan().all()


@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("at", [333, 715])
def test_a_value_out_of_range_in_a_late_tile(pp, size, bad, at):
    """V rows that only some rows of an item see, in tiles past the first turn of the rings."""
    call = _Call(pp, *size)
    clean, clean_lse = call()
    row = call.n - call.fresh + at
    call.vc[row // 16, row % 16, 1, 5] = bad
    out, lse = call()
    group = out.shape[1] // call.vc.shape[2]
    hit = torch.zeros(out.shape, dtype=torch.bool, device="cuda")
    hit[call.sees(row), group:2 * group, 5] = True
    assert torch.equal(out[~hit], clean[~hit]) and torch.equal(lse, clean_lse) and not clean.isnan().any()
    assert out[hit].isnan().all() if math.isnan(bad) else (out[hit] == bad).all()
