"""pp_kv_write8's slot maps: a block whose tokens do not stand next to one another is reported, in
whatever way they lie apart, and no map that keeps to the rule is, whatever calls were before it."""
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


class _Cache:
    def __init__(self, pp, blocks, block, heads=2, dim=64):
        self.block, self.heads, self.dim = block, heads, dim
        self.code = [torch.zeros((blocks, block, heads, dim), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2)]
        self.exp = [torch.zeros((blocks, heads), dtype=torch.int8, device="cuda") for _ in range(2)]
        self.pp, self.kv = pp, pp.KVCache.like(self.code[0])

    def write(self, slot):
        slot = torch.as_tensor(np.asarray(slot, np.int64), device="cuda")
        x = torch.randn((len(slot), self.heads, self.dim), device="cuda").to(torch.bfloat16)
        self.pp.pp_kv_write8(self.kv, x, x, slot, self.code[0], self.exp[0], self.code[1], self.exp[1])
        return x

    def reported(self):
        try:
            self.kv.sync()
        except self.pp.PPError as e:
            assert e.status == self.pp.PP_EBOUNDS
            return True
        return False


def _breaks(slot, blocks, block):
    """Whether some block's tokens do not stand next to one another: another block's between two of them, or 32 and
    more that are left out."""
    last, seen, at = None, set(), None
    for t, s in enumerate(slot):
        if s < 0 or s >= blocks * block:
            continue
        b = int(s) // block
        if b == last and t - at <= 32:
            at = t
            continue
        if b in seen:
            return True
        seen.add(b)
        last, at = b, t
    return False


def _run(b, first, n, block=16):
    return list(range(b * block + first, b * block + first + n))


APART = {
    "next to each other but for one": _run(3, 0, 1) + _run(5, 0, 1) + _run(3, 1, 1),
    "in turns": [s for i in range(16) for s in (3 * 16 + i, 5 * 16 + i)],
    "the last of a long call": _run(3, 0, 4) + [s for b in range(10, 260) for s in _run(b, 0, 16)] + _run(3, 4, 4),
    "32 left out between": _run(3, 0, 4) + [-1] * 32 + _run(3, 4, 4),
    "thousands left out between": _run(3, 0, 4) + [-1] * 5000 + _run(3, 4, 1),
    "among single ones": [b * 16 for b in range(10, 210)] + [100 * 16 + 1] + [b * 16 for b in range(210, 250)],
    "slots above the cache do not count": _run(3, 0, 1) + [1 << 40] * 40 + _run(3, 1, 1),
}


@pytest.mark.parametrize("name", APART)
def test_a_block_whose_tokens_lie_apart_is_reported(pp, name):
    c, slot = _Cache(pp, 300, 16), APART[name]
    assert _breaks(slot, 300, 16)
    with c.kv:
        for _ in range(3):
            c.write(slot)
            assert c.reported()
        c.write(_run(3, 0, 8) + _run(100, 0, 2))            # and nothing of it stays
        assert not c.reported()


NEXT = {
    "31 left out between": _run(3, 0, 4) + [-1] * 31 + _run(3, 4, 4) + _run(7, 0, 1),
    "in any order": [3 * 16 + x for x in (7, 2, 15, 0, 9)] + [5 * 16 + x for x in (1, 0)],
    "left out among others": [-1] * 100 + _run(3, 0, 16) + [-1] * 100 + _run(4, 0, 16),
}


@pytest.mark.parametrize("name", NEXT)
def test_a_map_that_keeps_to_the_rule_is_not(pp, name):
    c, slot = _Cache(pp, 300, 16), NEXT[name]
    assert not _breaks(slot, 300, 16)
    with c.kv:
        for _ in range(3):
            c.write(slot)
            assert not c.reported()


@pytest.mark.parametrize("block", [8, 64, 512])
def test_any_maps_after_one_another(pp, block):
    """Maps with the same blocks at other tokens, over one handle: only those that break the rule are reported, and what
    the others write is right."""
    rng = np.random.default_rng(block)
    blocks, seen = 40, set()
    c = _Cache(pp, blocks, block)
    with c.kv:
        for turn in range(40):
            slot = []
            for b in rng.permutation(blocks)[:rng.integers(1, blocks)]:
                slot += list(b * block + rng.permutation(block)[:rng.integers(1, block + 1)])
                slot += [-1] * int(rng.integers(0, 3) * rng.integers(0, 20))
            if turn % 2:                                    # one row of a block goes elsewhere
                i, j = rng.integers(0, len(slot), 2)
                slot.insert(int(j), slot.pop(int(i)))
            want = _breaks(slot, blocks, block)
            seen.add(want)
            # (every block anew, so that what it holds follows from this call)
            slot = np.asarray(slot)
            old = [(ref.values(x), e.cpu().numpy()) for x, e in zip(c.code, c.exp)]
            x = c.write(slot)
            assert c.reported() == want
            if not want and turn < 12:
                for (code, exp), got, e in zip(old, c.code, c.exp):
                    code, exp = ref.write8(x.double().cpu().numpy(), slot, code, exp, block)
                    assert np.array_equal(exp, e.cpu().numpy()) and np.array_equal(code, ref.values(got), equal_nan=True)
    assert seen == {False, True}


def test_a_captured_call_reports_what_its_map_holds_when_it_is_replayed(pp):
    c = _Cache(pp, 64, 16)
    good, bad = np.arange(200), np.concatenate([np.arange(100), [3], np.arange(112, 211)])
    slot = torch.tensor(good, device="cuda")
    x = torch.randn((200, 2, 64), device="cuda").to(torch.bfloat16)
    with c.kv:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            pp.pp_kv_write8(c.kv, x, x, slot, c.code[0], c.exp[0], c.code[1], c.exp[1])
        for m in (good, bad, good, bad, bad, good):
            slot.copy_(torch.tensor(m))
            graph.replay()
            assert c.reported() == (m is bad)


def test_layers_on_two_streams_at_once(pp):
    """One handle, two layers' caches, the same maps and others with the same blocks: none is reported, all are right."""
    rng = np.random.default_rng(3)
    block, blocks, h, dim = 16, 200, 2, 64
    maps = [np.concatenate([b * block + np.arange(block) for b in rng.permutation(blocks)]) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    layers = []
    for i in range(2):
        code = [torch.zeros((blocks, block, h, dim), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2)]
        exp = [torch.zeros((blocks, h), dtype=torch.int8, device="cuda") for _ in range(2)]
        rows = [torch.randn((blocks * block, h, dim), device="cuda").to(torch.bfloat16) for _ in range(2)]
        layers.append((rows, torch.tensor(maps[i], device="cuda"), code, exp))
    torch.cuda.synchronize()
    with pp.KVCache.like(layers[0][2][0]) as kv:
        for _ in range(50):
            for stream, (rows, slot, code, exp) in zip(streams, layers):
                pp.pp_kv_write8(kv, *rows, slot, code[0], exp[0], code[1], exp[1], stream=stream)
        for stream in streams:
            kv.sync(stream)
        for (rows, _, code, exp), slot in zip(layers, maps):
            for x, c, e in zip(rows, code, exp):
                want, we = ref.write8(x.double().cpu().numpy(), slot, np.zeros((blocks, block, h, dim)), np.zeros((blocks, h)), block)
                assert np.array_equal(we, e.cpu().numpy()) and np.array_equal(want, ref.values(c))
