"""Buffers of pp_kv_rotate and pp_kv_write8 that are given twice: an output that is another output, or
another one's input, is refused before anything is launched."""
import itertools

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

BF = torch.bfloat16


@pytest.fixture(scope="module")
def pp():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_01655_gb300 import build
    build.build()
    from paper_2608_01655_gb300 import binding
    return binding


def _refused(pp, call, **args):
    with pytest.raises(pp.PPError, match="PP_EINVAL"):
        call(**args)


def test_rotate(pp):
    # caches and rows of one shape, so that any of them can stand for any other
    some = {name: torch.full((16, 16, 2, 64), i + 1.0, dtype=BF, device="cuda") for i, name in enumerate(
        ("q", "k", "v", "q_out", "k_out", "k_cache", "v_cache"))}
    before = {name: t.clone() for name, t in some.items()}
    position, slot = torch.arange(16, dtype=torch.int32, device="cuda"), torch.arange(16, device="cuda")

    def run(**same):
        """same: buffers that are others, {name: other's}."""
        t = {name: some[same.get(name, name)] for name in some}
        rows = {name: (x if name.endswith("cache") else x[:, 0]) for name, x in t.items()}
        pp.pp_kv_rotate(kv, None, rows["q"], rows["k"], position, rows["q_out"], k_out=rows["k_out"], v=rows["v"], slot_map=slot,
                        k_cache=rows["k_cache"], v_cache=rows["v_cache"])

    outs, ins = ("q_out", "k_out", "k_cache", "v_cache"), ("q", "k", "v")
    with pp.KVCache.like(some["k_cache"]) as kv:
        for a, b in itertools.combinations(outs, 2):
            _refused(pp, run, **{a: b})
        for a, b in itertools.product(outs, ins):
            if (a, b) not in (("q_out", "q"), ("k_out", "k")):
                _refused(pp, run, **{a: b})
        kv.sync()
        for name, t in some.items():
            assert torch.equal(t, before[name])
        run(q_out="q", k_out="k")                           # in place
        run(k="q", v="q")                                   # one input for all
        run()
        kv.sync()
        # without queries their buffers are not looked at
        rows = {name: t[:, 0] for name, t in some.items()}
        assert pp._lib.pp_kv_rotate(kv.handle, 16, 0, rows["k"].data_ptr(), 0, 0, rows["k"].data_ptr(), 2048, 64, None, None, 1e-6,
                                    position.data_ptr(), 0, 0, None, 1.0, rows["k_out"].data_ptr(), 0, 0, rows["k_out"].data_ptr(),
                                    2048, 64, None, 0, 0, None, None, None, None) == pp.PP_OK
        kv.sync()


def test_write8(pp):
    code = [torch.zeros((4, 16, 2, 64), dtype=torch.float8_e4m3fn, device="cuda") for _ in range(2)]
    exp = [torch.zeros((4, 2), dtype=torch.int8, device="cuda") for _ in range(2)]
    x, slot = torch.ones((3, 2, 64), dtype=BF, device="cuda"), torch.arange(3, device="cuda")
    names = ("k_cache", "k_exp", "v_cache", "v_exp")
    place = dict(zip(names, (t.data_ptr() for pair in zip(code, exp) for t in pair)))
    with pp.KVCache.like(code[0]) as kv:
        def run(**same):
            at = [place[same.get(n, n)] for n in names]
            return pp._lib.pp_kv_write8(kv.handle, 3, x.data_ptr(), 128, 64, x.data_ptr(), 128, 64, slot.data_ptr(), *at, None)
        for a, b in itertools.combinations(names, 2):
            assert run(**{a: b}) == pp.PP_EINVAL and run(**{b: a}) == pp.PP_EINVAL
        kv.sync()
        assert not any(t.view(torch.uint8).any() for t in code + exp)
        assert run() == pp.PP_OK
        kv.sync()
        assert int(exp[0][0, 0]) == -8
