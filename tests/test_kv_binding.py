"""The binding of the paged cache's calls against a stand-in for the library: which tensors
reach it and on which stream.  No GPU."""
import types

import pytest

from paper_2608_01655_gb300 import build as ppbuild

torch = pytest.importorskip("torch")


class _Tensor:
    """What the binding looks at in a contiguous tensor on a device."""

    def __init__(self, shape, dtype, device=0):
        self.shape, self.dtype, self.index, self.is_cuda = torch.Size(shape), dtype, device, device >= 0
        self.device = f"cuda:{device}" if device >= 0 else "cpu"

    def get_device(self):
        return self.index

    def is_contiguous(self):
        return True

    def stride(self):
        st, n = [], 1
        for x in reversed(self.shape):
            st.insert(0, n)
            n *= x
        return tuple(st)

    def data_ptr(self):
        return 4096


@pytest.fixture
def pp(monkeypatch):
    ppbuild.build()
    from paper_2608_01655_gb300 import binding
    calls = []
    entry = lambda name: lambda *args: calls.append((name, args)) or 0
    names = ("pp_block_tables", "pp_kv_write", "pp_paged_attention", "pp_kv_destroy")
    monkeypatch.setattr(binding, "_lib", types.SimpleNamespace(**{n: entry(n) for n in names}))
    kv = binding.KVCache.__new__(binding.KVCache)
    kv._h, kv.shape, kv.strides, kv.dtype = 1, (4, 16, 2, 64), (2048, 128, 64), torch.bfloat16
    kv._i32, kv._i64, kv._f32, kv._device, kv._raw_stream = torch.int32, torch.int64, torch.float32, 0, lambda d: 0
    yield types.SimpleNamespace(module=binding, kv=kv, calls=calls)
    kv._h = None                                            # nothing to destroy


def _arguments():
    i32 = lambda *shape: _Tensor(shape, torch.int32)
    rows = lambda heads: _Tensor((3, heads, 64), torch.bfloat16)
    cache = lambda: _Tensor((4, 16, 2, 64), torch.bfloat16)
    slots = lambda: _Tensor((3,), torch.int64)
    return {
        "pp_block_tables": dict(length=i32(2), cached=i32(2), block_table=i32(2, 5), slot_map=slots(), position=i32(3),
                                q_start=i32(3), free_blocks=i32(7), free_head=i32(1), free_head_out=i32(1), node=i32(2),
                                chunk_map=i32(9, 4)),
        "pp_kv_write": dict(k=rows(2), v=rows(2), slot_map=slots(), k_cache=cache(), v_cache=cache()),
        "pp_paged_attention": dict(q=rows(4), k_cache=cache(), v_cache=cache(), block_table=i32(2, 5), q_start=i32(3),
                                   length=i32(2), max_q=2, out=rows(4), scale=0.1,
                                   lse=_Tensor((3, 4), torch.float32)),
    }


@pytest.mark.parametrize("call", ["pp_block_tables", "pp_kv_write", "pp_paged_attention"])
def test_tensors_of_another_device_are_refused(pp, call):
    """A tensor of another GPU, or of the host, is not taken for one of the handle's device."""
    fn = getattr(pp.module, call)
    fn(pp.kv, **_arguments()[call])
    assert len(pp.calls) == 1
    for name, value in _arguments()[call].items():
        if not isinstance(value, _Tensor):
            continue
        for device in (1, -1):
            args = _arguments()[call]
            args[name] = _Tensor(value.shape, value.dtype, device)
            with pytest.raises(ValueError, match=f"{name}: expected.*cuda:0"):
                fn(pp.kv, **args)
    assert len(pp.calls) == 1


class _Stream:
    def __init__(self, raw):
        self.cuda_stream = raw


def test_attention_on_another_stream_waits_for_the_last_one(pp, monkeypatch):
    """The scratch is one per handle: whoever comes from another stream is ordered after the last call."""
    waits = []
    monkeypatch.setattr(pp.module.KVCache, "_wait", lambda self, new, old: waits.append((new, old)) or True, raising=False)
    monkeypatch.setattr(pp.module._lib, "pp_kv_sync", lambda handle, stream: 0, raising=False)
    args = _arguments()
    call = lambda stream: pp.module.pp_paged_attention(pp.kv, **args["pp_paged_attention"], stream=stream)
    call(None)
    call(None)
    assert waits == []
    call(_Stream(5))
    assert waits == [(5, 0)]
    call(_Stream(5))
    call(7)
    call(None)
    assert waits == [(5, 0), (7, 5), (0, 7)]
    assert [a[-1].value or 0 if hasattr(a[-1], "value") else a[-1] for _, a in pp.calls] == [0, 0, 5, 5, 7, 0]
    # tables and writes use no scratch
    pp.module.pp_kv_write(pp.kv, **args["pp_kv_write"], stream=_Stream(9))
    pp.module.pp_block_tables(pp.kv, **args["pp_block_tables"], stream=_Stream(9))
    assert len(waits) == 3
    # a sync of another stream says nothing of the last call, one of its own that it has ended
    pp.kv.sync(_Stream(9))
    call(_Stream(5))
    assert waits[3:] == [(5, 0)]
    pp.kv.sync(_Stream(5))
    call(_Stream(7))
    assert len(waits) == 4


def test_captured_calls_are_not_followed(pp, monkeypatch):
    """_wait refuses while a stream is captured; the call to wait for stays the last one outside."""
    answers = iter([False, False, True])
    waits = []
    monkeypatch.setattr(pp.module.KVCache, "_wait", lambda self, new, old: waits.append((new, old)) or next(answers),
                        raising=False)
    call = lambda stream: pp.module.pp_paged_attention(pp.kv, **_arguments()["pp_paged_attention"], stream=stream)
    for raw in (3, 8, 8, 4):
        call(_Stream(raw))
    assert waits == [(8, 3), (8, 3), (4, 3)]
