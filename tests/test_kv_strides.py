"""Layouts whose rows lie over one another are refused before any CUDA call; others are not."""
import ctypes
import itertools

import numpy as np
import pytest

from paper_2608_01655_gb300 import build as ppbuild


@pytest.fixture(scope="module")
def pp():
    ppbuild.build()
    from paper_2608_01655_gb300 import binding
    return binding


def _create(pp, blocks, block_size, heads, dim, strides):
    h = ctypes.c_void_p(1)
    st = pp._lib.pp_kv_create(blocks, block_size, heads, dim, pp.PP_KV_BF16, *strides, None, ctypes.byref(h))
    if st == pp.PP_OK:
        pp._lib.pp_kv_destroy(h)
    return st


@pytest.mark.parametrize("blocks,block_size,heads,dim,strides", [
    (4, 16, 2, 64, (2048, 64, 64)),                     # a head's rows over the next token's
    (4, 16, 2, 64, (1024, 128, 64)),                    # blocks half over one another
    (4, 16, 2, 64, (64, 256, 128)),
    (4, 16, 8, 64, (1 << 20, 96, 64)),                  # rows that begin inside another
    (9, 8, 3, 8, (24, 16, 8)),
])
def test_create_refuses_overlapping_rows(pp, blocks, block_size, heads, dim, strides):
    assert _create(pp, blocks, block_size, heads, dim, strides) == pp.PP_EINVAL
    assert "overlap" in pp.last_error()


@pytest.mark.parametrize("blocks,block_size,heads,dim,strides", [
    (4, 16, 2, 64, (2048, 128, 64)), (4, 16, 2, 64, (2048, 64, 1024)), (4, 16, 2, 64, (64, 256, 4096)),
    (4, 16, 2, 64, (4096, 128, 64)),                    # K and V of a block in turn
    (4, 16, 1, 64, (1024, 64, 8 * 64)), (1, 16, 2, 64, (64, 128, 64)),         # an extent of 1: its stride says nothing
    (3, 8, 2, 8, (8, 48, 24)),                          # rows in the gaps of others
])
def test_create_takes_layouts_without_overlap(pp, blocks, block_size, heads, dim, strides):
    assert _create(pp, blocks, block_size, heads, dim, strides) != pp.PP_EINVAL       # no device here, or PP_OK


def test_overlap_against_all_pairs(pp):
    """Small layouts, each row's elements counted."""
    rng = np.random.default_rng(3)
    seen = {True: 0, False: 0}
    for _ in range(600):
        blocks, heads = (int(x) for x in rng.integers(1, 6, size=2))
        dim = int(rng.choice([8, 16, 24]))
        strides = [int(8 * x) for x in rng.integers(dim // 8, 40, size=3)]
        first = [b * strides[0] + t * strides[1] + h * strides[2]
                 for b, t, h in itertools.product(range(blocks), range(8), range(heads))]
        first.sort()
        overlap = any(b - a < dim for a, b in zip(first, first[1:]))
        refused = _create(pp, blocks, 8, heads, dim, strides) == pp.PP_EINVAL
        assert refused == overlap, (blocks, heads, dim, strides)
        seen[overlap] += 1
    assert min(seen.values()) > 50
