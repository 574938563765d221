"""One handle's attention calls from several streams, and its status read beside other work."""
import numpy as np
import pytest

from tests import kv_reference as ref

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


def test_one_handle_on_several_streams(pp):
    """Calls whose pieces are joined through the handle's scratch, by turns on three streams."""
    torch.manual_seed(14)
    kc, vc = (torch.randn((700, 16, 2, 128), device="cuda").to(torch.bfloat16) for _ in range(2))
    table = torch.arange(700, dtype=torch.int32, device="cuda")[None]
    calls = []
    for fresh, length in ((50, 11_000), (300, 10_000), (2, 11_200)):
        q = torch.randn((fresh, 8, 128), device="cuda").to(torch.bfloat16)
        calls.append((q, kc, vc, table, _i32([0, fresh]), _i32([length]), fresh))
    outs = []
    streams = [torch.cuda.Stream(), torch.cuda.default_stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    with pp.KVCache.like(kc) as kv:
        for turn in range(10):
            for i, call in enumerate(calls):
                out = torch.empty_like(call[0])
                torch.cuda.synchronize() if turn == 0 else None         # the first turn's calls have the GPU alone
                if turn % 2:
                    with torch.cuda.stream(streams[(turn + i) % 3]):
                        pp.pp_paged_attention(kv, *call, out, 0.1)
                else:
                    pp.pp_paged_attention(kv, *call, out, 0.1, stream=streams[(turn + i) % 3])
                outs.append(out)
        torch.cuda.synchronize()
        kv.sync()
    for i, (q, _, _, _, q_start, length, _) in enumerate(calls):
        want, _, tol, _ = ref.attention(q, kc, vc, table, q_start.tolist(), length.tolist(), 0.1, 0)
        assert ((outs[i].double() - want).abs() <= tol).all()
        for out in outs[i::3]:
            assert torch.equal(out.view(torch.int16), outs[i].view(torch.int16))


def test_an_eager_call_beside_a_capture(pp):
    """A capture takes the handle's calls after eager ones elsewhere, and eager ones go on during it."""
    torch.manual_seed(15)
    kc, vc = (torch.randn((200, 16, 2, 64), device="cuda").to(torch.float16) for _ in range(2))
    q = torch.randn((40, 4, 64), device="cuda").to(torch.float16)
    args = (q, kc, vc, torch.arange(200, dtype=torch.int32, device="cuda")[None], _i32([0, 40]), _i32([3000]), 40)
    first, captured, beside, after = (torch.empty_like(q) for _ in range(4))
    side = torch.cuda.Stream()
    with pp.KVCache.like(kc) as kv:
        pp.pp_paged_attention(kv, *args, first, 0.1)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, capture_error_mode="thread_local"):
            pp.pp_paged_attention(kv, *args, captured, 0.1)
            pp.pp_paged_attention(kv, *args, beside, 0.1, stream=side)
        side.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        pp.pp_paged_attention(kv, *args, after, 0.1, stream=side)
        kv.sync(side)
    for out in (captured, beside, after):
        assert torch.equal(out.view(torch.int16), first.view(torch.int16))


def test_sync_is_of_its_own_stream(pp):
    """Reading the status on a stream neither waits for work elsewhere nor leaves its clearing to it."""
    kc = torch.zeros((4, 16, 1, 8), dtype=torch.bfloat16, device="cuda")
    rows, wrong = torch.ones((1, 1, 8), dtype=torch.bfloat16, device="cuda"), torch.tensor([64], device="cuda")
    side, busy = torch.cuda.Stream(), torch.cuda.Event()
    with pp.KVCache.like(kc) as kv:
        pp.pp_kv_write(kv, rows, rows, wrong - 60, kc, kc.clone())
        torch.cuda.synchronize()
        torch.cuda._sleep(1_000_000_000)                    # half a second of the default stream
        busy.record()
        kv.sync(side)
        for _ in range(20):
            pp.pp_kv_write(kv, rows, rows, wrong, kc, kc, stream=side)
            with pytest.raises(pp.PPError, match="PP_EBOUNDS"):
                kv.sync(side)
        kv.sync(side)
        assert not busy.query()
        torch.cuda.synchronize()
