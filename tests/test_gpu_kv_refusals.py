"""Refusals of the paged cache's calls that need a handle."""
import pytest

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
    return torch.tensor(a, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("strides,overlap", [
    ((64, 64), True),                   # a token's second head over the next token's first
    ((256, 56), True), ((128, 64), True), ((8, 64), True),
    ((192, 128), True),                 # 2 x 192 = 3 x 128
    ((256, 64), False), ((300 * 8, 72), False),
    ((64, 64 * 5), False),              # tokens inside heads
    ((1600, 320), False)])
def test_output_rows_that_overlap_are_refused(pp, strides, overlap):
    kc, vc = (torch.randn((4, 16, 2, 64), device="cuda").to(torch.bfloat16) for _ in range(2))
    q = torch.randn((5, 4, 64), device="cuda").to(torch.bfloat16)
    base = torch.full((1 << 16,), 3.0, dtype=torch.bfloat16, device="cuda")
    out = base.as_strided(q.shape, (*strides, 1))
    args = (q, kc, vc, _i32([[2, 0, 3]]), _i32([0, 5]), _i32([40]), 5)
    with pp.KVCache.like(kc) as kv:
        if overlap:
            with pytest.raises(pp.PPError, match="overlap"):
                pp.pp_paged_attention(kv, *args, out, 0.125)
            kv.sync()
            assert (base == 3).all()
        else:
            want = torch.empty_like(q)
            pp.pp_paged_attention(kv, *args, out, 0.125)
            pp.pp_paged_attention(kv, *args, want, 0.125)
            kv.sync()
            assert torch.equal(out, want) and int((base != 3).sum()) <= q.numel()


def test_one_row_has_no_strides(pp):
    """An extent of 1 overlaps nothing, whatever its stride."""
    kc, vc = (torch.randn((4, 16, 1, 64), device="cuda").to(torch.bfloat16) for _ in range(2))
    q = torch.randn((3, 1, 64), device="cuda").to(torch.bfloat16)
    want, out = torch.empty_like(q), torch.empty_like(q).as_strided((3, 1, 64), (64, 8, 1))
    with pp.KVCache.like(kc) as kv:
        for o in (want, out):
            pp.pp_paged_attention(kv, q, kc, vc, _i32([[1, 2]]), _i32([0, 3]), _i32([20]), 3, o, 0.125)
        kv.sync()
    assert torch.equal(out, want)
