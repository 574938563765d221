"""The example's own comparison does not pass over NaN."""
import importlib.util
import os

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_01655_gb300 import build
    build.build()
    spec = importlib.util.spec_from_file_location("serve_prefixes", os.path.join(ROOT, "examples", "serve_prefixes.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("row", [0, 4])
def test_check_raises_where_the_output_is_not_finite(example, bad, row):
    layer, length, starts = example.Layer(), np.array([9, 7]), np.array([0, 2, 5])
    sequence = torch.arange(20, device="cuda").view(2, 10)
    out = torch.zeros((5, example.HEADS, example.DIM), dtype=torch.bfloat16, device="cuda")
    assert example.check(layer, sequence, length, starts, out, [0, 1]) == pytest.approx(1.0)
    out[row, 3, 5] = bad
    with pytest.raises(ArithmeticError):
        example.check(layer, sequence, length, starts, out, [0, 1])


def test_run_raises_where_the_attention_gives_nan(example, monkeypatch):
    real = example.pp.pp_paged_attention

    def broken(kv, q, k_cache, v_cache, table, q_start, length, max_q, out, scale):
        real(kv, q, k_cache, v_cache, table, q_start, length, max_q, out, scale)
        out.fill_(float("nan"))
    monkeypatch.setattr(example.pp, "pp_paged_attention", broken)
    with pytest.raises(ArithmeticError):
        example.run(requests=3, steps=1)
