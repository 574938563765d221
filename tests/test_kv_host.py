"""CPU checks of the paged cache's host side: the chunk map against walks of the
tree, and refusals that reach no CUDA call."""
import ctypes

import numpy as np
import pytest

from paper_2608_01655_gb300 import build as ppbuild


@pytest.fixture(scope="module")
def pp():
    ppbuild.build()
    from paper_2608_01655_gb300 import binding
    return binding


def _forest(rng, n, chain):
    parent = np.full(n, -1, np.int32)
    for i in range(1, n):
        parent[i] = i - 1 if rng.random() < chain else rng.integers(-1, i)
    perm = rng.permutation(n)
    out = np.full(n, -1, np.int32)
    out[perm] = np.where(parent < 0, -1, perm[parent])
    return out


def _closed(rng, parent, share):
    n = len(parent)
    res = np.zeros(n, np.uint8)
    done = np.zeros(n, bool)

    def visit(v):
        path = []
        while v >= 0 and not done[v]:
            path.append(v)
            v = parent[v]
        for u in reversed(path):
            res[u] = (parent[u] < 0 or res[parent[u]]) and rng.random() < share
            done[u] = True
    for v in range(n):
        visit(v)
    return res


def _walk(chunk_map, node):
    """Block ids of the resident chunks on the node's path, through the records,
    and the segments crossed."""
    rec = chunk_map
    cur = node if rec[node, 1] >= 0 else rec[node, 0]
    blocks, segments = [], 0
    top = None
    while cur >= 0:
        up, base, begin, end = (int(x) for x in rec[cur])
        assert base >= 0 and end > begin >= 0
        stop = end if top is None else min(end, top)
        blocks = [base + j - begin for j in range(begin, stop)] + blocks
        top, cur = begin, up
        segments += 1
    assert top in (None, 0)
    return blocks, segments


@pytest.mark.parametrize("n,chain,share,wmax,per", [(1, 0, 1, 1, 1), (2, 1, 1, 3, 4), (60, 0.5, 0.9, 3, 2),
                                                    (300, 0.9, 0.98, 1, 32), (400, 0.0, 0.7, 4, 16),
                                                    (500, 1.0, 1, 2, 8), (50, 0.5, 0.0, 1, 1)])
def test_chunk_map_walks(pp, n, chain, share, wmax, per):
    rng = np.random.default_rng(n)
    parent = _forest(rng, n, chain)
    weight = rng.integers(1, wmax + 1, size=n).astype(np.int32)
    res = _closed(rng, parent, share)
    rec, used = pp.pp_chunk_map(parent, weight, res, per)
    assert used == int((weight * res).sum()) * per
    owner = {}
    for v in range(n):
        path = []
        u = v
        while u >= 0:
            path.append(u)
            u = parent[u]
        path = [u for u in reversed(path) if res[u]]
        blocks, segments = _walk(rec, v)
        assert len(blocks) == sum(int(weight[u]) for u in path) * per
        assert segments <= np.log2(n + 1) + 1
        at = 0
        for u in path:                       # a chunk has the same blocks on every path, and no one else's
            own = tuple(blocks[at:at + int(weight[u]) * per])
            assert owner.setdefault(u, own) == own
            at += len(own)
    every = [b for own in owner.values() for b in own]
    assert sorted(every) == list(range(used))


def test_chunk_map_empty(pp):
    rec, used = pp.pp_chunk_map(np.zeros(0), np.zeros(0), np.zeros(0), 4)
    assert rec.shape == (0, 4) and used == 0


@pytest.mark.parametrize("parent,weight,resident,per,status", [
    ([1, 0], [1, 1], [0, 0], 1, "PP_ENOTTREE"),          # a cycle
    ([0], [1], [1], 1, "PP_ENOTTREE"),
    ([5], [1], [1], 1, "PP_ENOTTREE"),
    ([-2], [1], [1], 1, "PP_ENOTTREE"),
    ([-1, 0], [1, 1], [0, 1], 1, "PP_EINVAL"),           # not closed under parents
    ([-1], [0], [1], 1, "PP_EINVAL"),
    ([-1], [1], [1], 0, "PP_EINVAL"),
    ([-1, -1], [1 << 20, 1 << 20], [1, 1], 1 << 20, "PP_EOVERFLOW"),
])
def test_chunk_map_refusals(pp, parent, weight, resident, per, status):
    with pytest.raises(pp.PPError, match=status):
        pp.pp_chunk_map(parent, weight, resident, per)


def test_chunk_map_null(pp):
    used = ctypes.c_int32(0)
    assert pp._lib.pp_chunk_map(1, None, None, None, 1, None, ctypes.byref(used)) == pp.PP_EINVAL
    assert pp._lib.pp_chunk_map(-1, None, None, None, 1, None, ctypes.byref(used)) == pp.PP_EINVAL
    assert pp._lib.pp_chunk_map(0, None, None, None, 1, None, None) == pp.PP_EINVAL


@pytest.mark.parametrize("kw", [dict(blocks=0), dict(blocks=(1 << 30) + 1), dict(block_size=0), dict(block_size=4),
                                dict(block_size=24), dict(block_size=1024), dict(kv_heads=0), dict(head_dim=0),
                                dict(head_dim=12), dict(head_dim=136), dict(dtype=2), dict(dtype=-1),
                                dict(strides=(0, 128, 64)), dict(strides=(4096, 130, 64)),
                                dict(strides=(4096, 128, -64)), dict(strides=(4096, 56, 64)),
                                dict(strides=(1 << 38, 128, 64))])
def test_create_refusals(pp, kw):
    a = dict(blocks=4, block_size=16, kv_heads=2, head_dim=64, dtype=pp.PP_KV_BF16, strides=(0, 0, 0))
    a.update(kw)
    h = ctypes.c_void_p(1)
    st = pp._lib.pp_kv_create(a["blocks"], a["block_size"], a["kv_heads"], a["head_dim"], a["dtype"], *a["strides"],
                              None, ctypes.byref(h))
    assert st == pp.PP_EINVAL and h.value is None
    assert pp.last_error()


def test_null_handles(pp):
    assert pp._lib.pp_kv_create(4, 16, 2, 64, 0, 0, 0, 0, None, None) == pp.PP_EINVAL
    assert pp._lib.pp_kv_destroy(None) == pp.PP_OK
    assert pp._lib.pp_kv_sync(None, None) == pp.PP_EINVAL
    assert pp._lib.pp_kv_write(*[0 if t in (ctypes.c_int32, ctypes.c_int64) else None
                                 for t in pp._SIGS["pp_kv_write"]]) == pp.PP_EINVAL
