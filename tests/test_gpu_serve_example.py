"""The example runs a plan, the cache's tables, writes and attention together."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_serve_prefixes():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_01655_gb300 import build
    build.build()
    spec = importlib.util.spec_from_file_location("serve_prefixes", os.path.join(ROOT, "examples", "serve_prefixes.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    result = example.run(requests=10, steps=2)
    assert 0 < result["cached_tokens"] < result["prompt_tokens"]
    # weights, outputs and their 16-bit roundings: 2^-8 each of the largest value at most
    assert result["worst_error"] < 2 * 2.0 ** -8
