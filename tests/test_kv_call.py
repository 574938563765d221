"""The extension that makes the cache's calls: conversions, refusals, and the same tensor checks as the binding has in
Python.  No GPU."""
import ctypes
import itertools

import pytest

from paper_2608_01655_gb300 import build as ppbuild

torch = pytest.importorskip("torch")

CALLS = ("pp_block_tables", "pp_kv_write", "pp_paged_attention", "pp_kv_rotate", "pp_kv_write8", "pp_paged_attention8")
ZERO = {ctypes.c_int32: 0, ctypes.c_int64: 0, ctypes.c_float: 0.0, ctypes.c_size_t: 0}


@pytest.fixture(scope="module")
def pp():
    ppbuild.build()
    from paper_2608_01655_gb300 import binding
    if binding._fast is None:
        pytest.skip("built without Python's headers")
    return binding


@pytest.mark.parametrize("name", CALLS)
def test_calls_go_to_the_library(pp, name):
    """With a null handle every call is refused by the library, whatever stands for the null pointers."""
    call = getattr(pp._lib, name)
    assert call is getattr(pp._fast, name)
    for null in (None, 0, ctypes.c_void_p(0), ctypes.c_void_p(None)):
        assert call(*[ZERO.get(t, null) for t in pp._SIGS[name]]) == pp.PP_EINVAL
        assert "null cache handle" in pp.last_error()


@pytest.mark.parametrize("name", CALLS)
def test_arguments_of_other_types_or_sizes_are_refused(pp, name):
    call, good = getattr(pp._lib, name), [ZERO.get(t) for t in pp._SIGS[name]]
    for args in (good[:-1], good + [0], []):
        with pytest.raises(TypeError, match="arguments"):
            call(*args)
    for k, t in enumerate(pp._SIGS[name]):
        bad = ["x", 1.5, 1 << 70] if t is not ctypes.c_float else ["x", None]
        if t is ctypes.c_int32:
            bad += [1 << 31, -(1 << 31) - 1, None]
        if t is ctypes.c_int64:
            bad += [1 << 63, None]
        for x in bad:
            with pytest.raises((TypeError, OverflowError, AttributeError)):
                call(*good[:k], x, *good[k + 1:])


def test_binding_to_another_signature_is_refused(pp):
    with pytest.raises(TypeError, match="takes"):
        pp._fast.bind("pp_kv_write", "pip", 1)
    with pytest.raises(ValueError, match="no call"):
        pp._fast.bind("pp_kv_sync", "pp", 1)


def _handle(pp, stored=None):
    kv = pp.KVCache.__new__(pp.KVCache)
    kv._h, kv.shape, kv.strides, kv.dtype, kv._device = None, (4, 16, 2, 64), (2048, 128, 64), torch.bfloat16, -1
    if stored:
        kv._stored = stored
    return kv


def _both(pp, monkeypatch, f):
    out = []
    for fast in (pp._fast, None):
        with monkeypatch.context() as m:
            m.setattr(pp, "_fast", fast)
            try:
                out.append(f())
            except ValueError as e:
                out.append(str(e))
    assert out[0] == out[1]
    return out[0]


def test_checks_are_those_in_python(pp, monkeypatch):
    """Tensors of the host (device -1 here), right and wrong in every way, through both."""
    kv, right = _handle(pp), 0
    base = torch.zeros(1 << 16, dtype=torch.bfloat16)
    for tokens, heads, dim in itertools.product((0, 1, 3), (1, 2), (64, 32)):
        for strides in ((128, 64, 1), (256, 64, 1), (64, 7, 1), (128, 64, 2), (1, 1, 1)):
            for dtype in (torch.bfloat16, torch.float16):
                t = base.view(dtype).as_strided((tokens, heads, dim), strides)
                for want in ((tokens, heads), (tokens + 1, heads), (3, 2)):
                    right += isinstance(_both(pp, monkeypatch, lambda: kv._rows(t, "t", *want)), tuple)
    assert right > 20
    assert isinstance(_both(pp, monkeypatch, lambda: kv._rows(base, "t", 1, 1)), str)           # one dimension
    for t in (base[:5], base[:10:2], base[:5].float(), base[:4], base[:5].view(1, 5)):
        _both(pp, monkeypatch, lambda: kv._arg(t, "t", torch.bfloat16, (5,)))
    for handle, dtype in ((kv, torch.bfloat16), (_handle(pp, torch.float8_e4m3fn), torch.float8_e4m3fn)):
        for shape in ((4, 16, 2, 64), (1, 16, 2, 64), (4, 16, 1, 64), (4, 16, 2, 32)):
            for strides in ((2048, 128, 64, 1), (4096, 128, 64, 1), (2048, 64, 1024, 1), (7, 128, 64, 1), (2048, 128, 9, 1), (2048, 128, 64, 2)):
                for mine in ((4, 16, 2, 64), (1, 16, 2, 64), (4, 16, 1, 64)):
                    handle.shape = mine
                    t = torch.zeros(1 << 16, dtype=dtype).as_strided(shape, strides)
                    got = _both(pp, monkeypatch, lambda: handle._cache(t, "t"))
                    assert isinstance(got, (int, str))
    kv._device = 0
    assert isinstance(_both(pp, monkeypatch, lambda: kv._rows(torch.zeros((3, 2, 64), dtype=torch.bfloat16), "t", 3, 2)), str)


def test_things_that_are_no_tensors(pp):
    for f in (lambda x: pp._fast.rows(x, None, 1, 1, 1, 0), lambda x: pp._fast.contiguous(x, None, (1,), 0),
              lambda x: pp._fast.cache(x, None, (1,) * 4, (1,) * 3, 0)):
        for x in (None, 3, "t"):
            with pytest.raises(AttributeError):
                f(x)
    for f in (pp._fast.rows, pp._fast.contiguous, pp._fast.cache):
        with pytest.raises(TypeError):
            f(1)
