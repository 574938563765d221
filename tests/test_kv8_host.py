"""Host parts of the rotation and of the 8-bit cache: frequencies, fractions of a turn, refusals
without a handle, and which tensors the binding lets through.  No GPU."""
import ctypes
import math
import types
from fractions import Fraction

import numpy as np
import pytest

from paper_2608_01655_gb300 import build as ppbuild
from tests import kv8_reference as ref
from tests.test_kv_binding import _Tensor

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def lib():
    ppbuild.build()
    from paper_2608_01655_gb300 import binding
    return binding


def _frequencies(lib, pairs, base=10000.0, factor=1.0, original=0.0, slow=1.0, fast=32.0):
    out = np.full(max(pairs, 1), 7.0)
    st = lib._lib.pp_rotary_frequencies(pairs, base, factor, original, slow, fast, out.ctypes.data_as(ctypes.c_void_p))
    assert st == lib.PP_OK, lib.last_error()
    return out[:pairs]


@pytest.mark.parametrize("pairs", [0, 1, 5, 32, 64])
@pytest.mark.parametrize("base", [10000.0, 500000.0, 3.0])
def test_frequencies(lib, pairs, base):
    i = np.arange(pairs)
    want = np.array([math.exp(-math.log(base) * x / pairs) for x in i])
    assert np.allclose(_frequencies(lib, pairs, base), want, rtol=1e-14, atol=0)
    assert np.allclose(_frequencies(lib, pairs, base, 8.0), want / 8, rtol=1e-14, atol=0)


@pytest.mark.parametrize("original,slow,fast", [(8192, 1, 32), (32768, 1, 4), (100, 0, 0.5)])
def test_frequencies_by_parts(lib, original, slow, fast):
    plain = _frequencies(lib, 64)
    got = _frequencies(lib, 64, factor=16.0, original=original, slow=slow, fast=fast)
    for f, g in zip(plain, got):
        turns = original * f / (2 * math.pi)
        if turns >= fast:
            assert g == pytest.approx(f, rel=1e-14)
        elif turns <= slow:
            assert g == pytest.approx(f / 16, rel=1e-14)
        else:
            keep = (turns - slow) / (fast - slow)
            assert g == pytest.approx(f * keep + f / 16 * (1 - keep), rel=1e-13)
    assert (np.diff(got) < 0).all()


def test_turns(lib):
    """Each is the frequency over 2 pi modulo 1, to 53 bits."""
    f = np.array([1.0, 1e-4, 0.5, 2 * math.pi, 7.0, 1e9, -1.0, -1e-30, 0.0, 1e-18])
    out = np.zeros(len(f), np.uint64)
    assert lib._lib.pp_rotary_turns(len(f), f.ctypes.data_as(ctypes.c_void_p), out.ctypes.data_as(ctypes.c_void_p)) == lib.PP_OK
    two_pi = Fraction("6.28318530717958647692528676655900576839433879875021")
    for x, got in zip(f, out):
        exact = Fraction(float(x)) / two_pi
        off = Fraction(int(got), 1 << 64) - exact
        off -= round(off)                                   # whole turns do not matter
        assert abs(off) <= abs(exact) * Fraction(1, 1 << 51) + Fraction(1, 1 << 53)


@pytest.mark.parametrize("args", [(-1, 1e4, 1, 0, 1, 2), (65, 1e4, 1, 0, 1, 2), (4, 0, 1, 0, 1, 2), (4, -2, 1, 0, 1, 2),
                                  (4, math.inf, 1, 0, 1, 2), (4, math.nan, 1, 0, 1, 2), (4, 1e4, 0, 0, 1, 2),
                                  (4, 1e4, math.nan, 0, 1, 2), (4, 1e4, 1, -1, 1, 2), (4, 1e4, 1, math.inf, 1, 2),
                                  (4, 1e4, 1, 9, 2, 2), (4, 1e4, 1, 9, math.nan, 2)])
def test_frequency_refusals(lib, args):
    out = np.full(64, 7.0)
    assert lib._lib.pp_rotary_frequencies(*args, out.ctypes.data_as(ctypes.c_void_p)) == lib.PP_EINVAL
    assert (out == 7).all() and lib.last_error()


def test_turn_refusals(lib):
    f, out = np.array([1.0, math.inf]), np.zeros(2, np.uint64)
    P = lambda a: a.ctypes.data_as(ctypes.c_void_p)
    turns = lib._lib.pp_rotary_turns
    assert turns(2, P(f), P(out)) == lib.PP_EINVAL and not out.any()
    assert turns(1, None, P(out)) == lib.PP_EINVAL and turns(1, P(f), None) == lib.PP_EINVAL
    assert turns(-1, P(f), P(out)) == lib.PP_EINVAL and turns(65, P(f), P(out)) == lib.PP_EINVAL
    assert turns(0, None, None) == lib.PP_OK
    assert lib._lib.pp_rotary_frequencies(0, 1e4, 1, 0, 1, 2, None) == lib.PP_OK
    assert lib._lib.pp_rotary_frequencies(1, 1e4, 1, 0, 1, 2, None) == lib.PP_EINVAL


@pytest.mark.parametrize("name", ["pp_kv_rotate", "pp_kv_write8", "pp_kv_workspace", "pp_paged_attention8"])
def test_null_handles(lib, name):
    zero = {ctypes.c_int32: 0, ctypes.c_int64: 0, ctypes.c_float: 0.0, ctypes.c_size_t: 0}
    assert getattr(lib._lib, name)(*[zero.get(t) for t in lib._SIGS[name]]) == lib.PP_EINVAL
    assert "null cache handle" in lib.last_error()


@pytest.mark.parametrize("kw", [dict(head_dim=8), dict(head_dim=72), dict(head_dim=136), dict(strides=(4096, 136, 64)),
                                dict(strides=(4096, 128, 72)), dict(strides=(4104, 128, 64)), dict(strides=(2048, 64, 64)),
                                dict(block_size=4)])
@pytest.mark.parametrize("dtype", ["PP_KV_BF16_E4M3", "PP_KV_F16_E4M3"])
def test_create_refusals_of_8_bit_layouts(lib, kw, dtype):
    a = dict(blocks=4, block_size=16, kv_heads=2, head_dim=64, strides=(0, 0, 0))
    a.update(kw)
    h = ctypes.c_void_p(1)
    st = lib._lib.pp_kv_create(a["blocks"], a["block_size"], a["kv_heads"], a["head_dim"], getattr(lib, dtype),
                               *a["strides"], None, ctypes.byref(h))
    assert st == lib.PP_EINVAL and h.value is None and lib.last_error()


def test_rotary_arguments(lib):
    for kw in (dict(rotated=3), dict(rotated=-2), dict(rotated=4, frequencies=[1.0]), dict(rotated=4, frequencies=[[1.0, 2.0]])):
        with pytest.raises(ValueError):
            lib.Rotary(**kw)
    with pytest.raises(lib.PPError, match="PP_EINVAL"):
        lib.Rotary(130)
    with pytest.raises(lib.PPError, match="PP_EINVAL"):
        lib.Rotary(4, frequencies=[1.0, math.nan])


# ---------------------------------------------------------------------------
# the binding, against a stand-in for the library
# ---------------------------------------------------------------------------
CALLS = ("pp_kv_rotate", "pp_kv_write8", "pp_paged_attention8")


@pytest.fixture(params=["extension", "Python"])
def pp(lib, monkeypatch, request):
    """The binding's checks, of the extension module and of the binding itself."""
    if request.param == "Python":
        monkeypatch.setattr(lib, "_fast", None)
    calls = []
    entry = lambda name: lambda *args: calls.append((name, args)) or 0
    monkeypatch.setattr(lib, "_lib", types.SimpleNamespace(**{n: entry(n) for n in CALLS + ("pp_kv_write", "pp_kv_destroy")}))
    made = []

    def handle(eight):
        kv = lib.KVCache.__new__(lib.KVCache)
        kv._h, kv.shape, kv.strides, kv.dtype = 1, (4, 16, 2, 64), (2048, 128, 64), torch.bfloat16
        kv._i32, kv._i64, kv._f32, kv._device, kv._raw_stream = torch.int32, torch.int64, torch.float32, 0, lambda d: 0
        if eight:
            kv._stored, kv._i8, kv._u8 = torch.float8_e4m3fn, torch.int8, torch.uint8
        made.append(kv)
        return kv

    yield types.SimpleNamespace(module=lib, handle=handle, calls=calls)
    for kv in made:
        kv._h = None                                        # nothing to destroy


def _arguments():
    i32 = lambda *shape: _Tensor(shape, torch.int32)
    rows = lambda heads: _Tensor((3, heads, 64), torch.bfloat16)
    cache = lambda: _Tensor((4, 16, 2, 64), torch.float8_e4m3fn)
    wide = lambda: _Tensor((4, 16, 2, 64), torch.bfloat16)
    exps = lambda: _Tensor((4, 2), torch.int8)
    slots = lambda: _Tensor((3,), torch.int64)
    weight = lambda: _Tensor((64,), torch.bfloat16)
    rotary = types.SimpleNamespace(rotated=32, interleaved=0, amplitude=1.0, _ptr=4096, _device=0)
    return {
        "pp_kv_rotate": dict(rotary=rotary, q=rows(4), k=rows(2), position=i32(3), q_out=rows(4), k_out=rows(2),
                             q_weight=weight(), k_weight=weight(), v=rows(2), slot_map=slots(), k_cache=wide(), v_cache=wide()),
        "pp_kv_write8": dict(k=rows(2), v=rows(2), slot_map=slots(), k_cache=cache(), k_exp=exps(), v_cache=cache(),
                             v_exp=exps()),
        "pp_paged_attention8": dict(q=rows(4), k_cache=cache(), k_exp=exps(), v_cache=cache(), v_exp=exps(),
                                    block_table=i32(2, 5), q_start=i32(3), length=i32(2), max_q=2, out=rows(4), scale=0.1,
                                    lse=_Tensor((3, 4), torch.float32), workspace=_Tensor((1 << 20,), torch.uint8)),
    }


@pytest.mark.parametrize("call", CALLS)
def test_tensors_of_another_device_type_or_shape_are_refused(pp, call):
    fn, kv = getattr(pp.module, call), pp.handle(call != "pp_kv_rotate")
    fn(kv, **_arguments()[call])
    assert len(pp.calls) == 1
    for name, value in _arguments()[call].items():
        if not isinstance(value, _Tensor):
            continue
        longer = tuple(value.shape[:-1]) + (value.shape[-1] + 16,)
        wrong = [_Tensor(value.shape, value.dtype, 1), _Tensor(value.shape, value.dtype, -1),
                 _Tensor(value.shape, torch.float64)]
        # shapes that others are measured by are not wrong by themselves
        if name not in ("workspace", "block_table", "slot_map", "position", "length"):
            wrong.append(_Tensor(longer, value.dtype))
        for bad in wrong:
            args = _arguments()[call]
            args[name] = bad
            with pytest.raises(ValueError, match=f"{name}: expected"):
                fn(kv, **args)
    assert len(pp.calls) == 1


def test_handles_of_the_other_kind_are_refused(pp):
    for call in ("pp_kv_write8", "pp_paged_attention8"):
        with pytest.raises(ValueError, match="eight_bit"):
            getattr(pp.module, call)(pp.handle(False), **_arguments()[call])
    args = {k: v for k, v in _arguments()["pp_kv_write8"].items() if not k.endswith("_exp")}
    with pytest.raises(ValueError, match="k_cache: expected a torch.float8_e4m3fn"):
        wide = _Tensor((4, 16, 2, 64), torch.bfloat16)
        pp.module.pp_kv_write(pp.handle(True), **{**args, "k_cache": wide, "v_cache": wide})
    assert not pp.calls


def test_rotary_of_another_device_or_width_is_refused(pp):
    for change in (dict(_device=1), dict(rotated=80)):
        args = _arguments()["pp_kv_rotate"]
        for k, v in change.items():
            setattr(args["rotary"], k, v)
        with pytest.raises(ValueError, match="rotary:"):
            pp.module.pp_kv_rotate(pp.handle(False), **args)
    args = _arguments()["pp_kv_rotate"]
    args["q"] = None
    with pytest.raises(ValueError, match="q and q_out"):
        pp.module.pp_kv_rotate(pp.handle(False), **args)
    assert not pp.calls


def test_attention8_on_another_stream_waits_for_the_last_one(pp, monkeypatch):
    waits = []
    monkeypatch.setattr(pp.module.KVCache, "_wait", lambda self, new, old: waits.append((new, old)) or True)
    kv = pp.handle(True)
    for raw in (5, 5, 7):
        pp.module.pp_paged_attention8(kv, **_arguments()["pp_paged_attention8"], stream=raw)
    assert waits == [(7, 5)]


# ---------------------------------------------------------------------------
# the reference itself
# ---------------------------------------------------------------------------
def test_reference_codes_are_those_of_the_type():
    """Every e4m3 number is its own nearest, and halves between neighbours go to the even one."""
    code = torch.arange(256, dtype=torch.uint8)
    all_ = ref.values(code)
    finite = all_[np.isfinite(all_)]
    assert len(finite) == 254 and np.array_equal(ref.e4m3(finite), finite)
    up = np.unique(finite)
    middle = (up[1:] + up[:-1]) / 2
    want = torch.tensor(middle).float().to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(ref.e4m3(middle), want)
    assert ref.e4m3(1e9) == 448 and np.isnan(ref.e4m3(np.nan))


def test_reference_bound_sees_a_mistake():
    """A V exponent that is off by one, or a mask by one key, is far outside the bound."""
    torch.manual_seed(0)
    kc, ke = ref.to8(torch.randn(6, 16, 1, 32))
    vc, ve = ref.to8(torch.randn(6, 16, 1, 32))
    q = torch.randn(2, 2, 32).to(torch.bfloat16)
    table = torch.tensor([[3, 0, 5, 1]])
    for direct in (True, False):
        args = (q, kc, ke, vc, ve, table, [0, 2], [50], 0.2, 0)
        out, lse, tol, ltol = ref.attention8(*args, direct)
        other = ref.attention8(q, kc, ke, vc, ve + 1, table, [0, 2], [50], 0.2, 0, direct)[0]
        assert ((other - out).abs() > tol).float().mean() > 0.9
        other, olse = ref.attention8(q, kc, ke, vc, ve, table, [0, 2], [49], 0.2, 0, direct)[:2]
        assert ((other - out).abs() > tol).float().mean() > 0.5 and ((olse - lse).abs() > ltol).all()
