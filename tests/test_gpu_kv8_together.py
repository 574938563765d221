"""The operators of an 8-bit cache as a program uses them: block tables, rotation, write and attention, step after
step, chunks first and single tokens then, the latter also captured in a graph and replayed."""
import importlib.util
import math
import os

import numpy as np
import pytest

from tests import kv8_reference as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


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


@pytest.mark.parametrize("heads,kv_heads,dim,block,dtype", [(8, 2, 128, 16, torch.bfloat16), (6, 3, 80, 32, torch.float16),
                                                            (4, 4, 64, 8, torch.bfloat16)])
@pytest.mark.parametrize("graph", [False, True])
def test_steps(pp, heads, kv_heads, dim, block, dtype, graph):
    torch.manual_seed(dim)
    requests, width, steps = 5, 24, 6
    prompt = np.array([1, block, 3 * block + 5, 100, 37])
    length, cached = _i32(prompt), _i32([0] * requests)
    blocks = requests * width
    code = [torch.randint(0, 256, (blocks, block, kv_heads, dim), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
            for _ in range(2)]
    exp = [torch.randint(-128, 128, (blocks, kv_heads), dtype=torch.int8, device="cuda") for _ in range(2)]
    want = [(ref.values(c), e.cpu().numpy()) for c, e in zip(code, exp)]
    table, free = torch.full((requests, width), -1, dtype=torch.int32, device="cuda"), torch.randperm(blocks, device="cuda").int()
    head, head_out = _i32([0]), _i32([0])
    q_start = _i32([0] * (requests + 1))
    rotary = pp.Rotary(dim // 16 * 8, factor=4.0, original=64, amplitude=1.1)
    weight = (torch.rand(dim, device="cuda") + 0.5).to(dtype)
    scale = dim ** -0.5
    with pp.KVCache.like(code[0], dtype=dtype) as kv:
        workspace = torch.empty(kv.workspace_size(requests, width, blocks), dtype=torch.uint8, device="cuda")

        def buffers(tokens):
            qkv = torch.empty((tokens, heads + 2 * kv_heads, dim), dtype=dtype, device="cuda")
            return dict(qkv=qkv, slot=torch.empty(tokens, dtype=torch.int64, device="cuda"), position=_i32([0] * tokens),
                        out=torch.empty((tokens, heads, dim), dtype=dtype, device="cuda"),
                        lse=torch.empty((tokens, heads), device="cuda"))

        def step(b, max_q):
            q, k, v = b["qkv"].split((heads, kv_heads, kv_heads), 1)
            pp.pp_block_tables(kv, length, cached, table, b["slot"], b["position"], q_start, free, head, head_out)
            pp.pp_kv_rotate(kv, rotary, q, k, b["position"], q, k_out=k, q_weight=weight, k_weight=weight)    # in place
            pp.pp_kv_write8(kv, k, v, b["slot"], code[0], exp[0], code[1], exp[1])
            pp.pp_paged_attention8(kv, q, code[0], exp[0], code[1], exp[1], table, q_start, length, max_q, b["out"], scale,
                                   lse=b["lse"], workspace=workspace)
            head.copy_(head_out)

        def check(b, raw, fresh, max_q):
            nonlocal want
            kv.sync()
            tokens = int(sum(fresh))
            assert q_start.tolist() == [0] + np.cumsum(fresh).tolist()
            q, k, v = b["qkv"].split((heads, kv_heads, kv_heads), 1)
            for got, was in ((q, raw[0]), (k, raw[1])):
                y, tol = ref.rotate(was, weight, 1e-6, b["position"], rotary.frequencies, rotary.rotated, False, 1.1)
                assert ((got.double() - y).abs() <= tol)[:tokens].all()
            slot = b["slot"].cpu().numpy()
            want = [ref.write8(x.double().cpu().numpy(), slot, *w, block) for x, w in zip((k, v), want)]
            for c, e, (wc, we) in zip(code, exp, want):
                got = ref.values(c)
                assert np.array_equal(e.cpu().numpy(), we) and ((got == wc) | (np.isnan(got) & np.isnan(wc))).all()
            direct = max_q * (heads // kv_heads) <= 48
            o, l, tol, ltol = ref.attention8(q[:tokens], code[0], exp[0], code[1], exp[1], table, q_start.tolist(), length.tolist(),
                                             scale, 0, direct)
            assert ((b["out"][:tokens].double() - o).abs() <= tol).all()
            assert ((b["lse"][:tokens].double() - l).abs() <= ltol).all()

        # the prompts in one step; its buffers are padded
        b = buffers(int(prompt.sum()) + 9)
        b["qkv"].normal_()
        raw = [x.clone() for x in b["qkv"].split((heads, kv_heads, kv_heads), 1)]
        step(b, int(prompt.max()))
        check(b, raw, prompt, int(prompt.max()))
        # then a token each
        b = buffers(requests)
        g = None
        if graph:
            b["qkv"].normal_()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                step(b, 1)
        for _ in range(steps):
            cached.copy_(length)
            length += 1
            b["qkv"].normal_().mul_(2.0 ** float(np.random.default_rng(int(length[0])).integers(-3, 4)))
            raw = [x.clone() for x in b["qkv"].split((heads, kv_heads, kv_heads), 1)]
            if g:
                g.replay()
            else:
                step(b, 1)
            check(b, raw, [1] * requests, 1)


def test_example_with_an_8_bit_cache(pp):
    spec = importlib.util.spec_from_file_location("serve_prefixes", os.path.join(ROOT, "examples", "serve_prefixes.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    result = example.run(requests=10, steps=2, eight_bit=True)
    assert 0 < result["cached_tokens"] < result["prompt_tokens"] and math.isfinite(result["worst_error"])
