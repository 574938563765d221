"""Bounded waits of the attention kernel: copies that are waited for and never come.  The
launch ends with PP_ETIMEOUT in the status word, nothing is left behind, and calls queued
behind it without a sync between are right."""
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


# a tile a CTA; items in many pieces, joined in shares; several tiles and items a CTA
@pytest.mark.parametrize("fresh,length,kv_heads", [([40, 70], [100, 300], 2), ([40], [20_000], 2), ([600, 300], [1500, 700], 8)])
@pytest.mark.parametrize("dim,dtype", [(128, torch.bfloat16), (64, torch.float16)])
def test_a_wait_that_runs_out_ends_the_launch(pp, fresh, length, kv_heads, dim, dtype):
    torch.manual_seed(16)
    need = [-(-n // 16) for n in length]
    kc, vc = (torch.randn((sum(need), 16, kv_heads, dim), device="cuda").to(dtype) for _ in range(2))
    table, at = np.zeros((len(fresh), max(need))), 0
    for r, n in enumerate(need):
        table[r, :n] = np.arange(at, at + n)
        at += n
    q = torch.randn((sum(fresh), 2 * kv_heads, dim), device="cuda").to(dtype)
    q_start = np.concatenate([[0], np.cumsum(fresh)])
    args = (q, kc, vc, _i32(table), _i32(q_start), _i32(length), max(fresh))
    lost, behind, after = (torch.full_like(q, 7) for _ in range(3))
    with pp.KVCache.like(kc) as kv:
        try:
            pp.pp_test_inject(2, 1)
            pp.pp_paged_attention(kv, *args, lost, 0.1)
        finally:
            pp.pp_test_inject(2, -1)
        pp.pp_paged_attention(kv, *args, behind, 0.1)
        with pytest.raises(pp.PPError) as e:
            kv.sync()
        assert e.value.status == pp.PP_ETIMEOUT
        kv.sync()
        pp.pp_paged_attention(kv, *args, after, 0.1)
        kv.sync()
    want, _, tol, _ = ref.attention(q, kc, vc, args[3], q_start, length, 0.1, 0)
    assert ((behind.double() - want).abs() <= tol).all()
    assert torch.equal(after.view(torch.int16), behind.view(torch.int16))
