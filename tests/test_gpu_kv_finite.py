"""Attention in graphs, in wider output buffers, in many pieces and on two streams, compared
so that a NaN fails: every element has to lie within the bound, out and lse alike."""
import math

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


class _Step:
    """Requests over blocks of their own in any order; out and lse start as NaN."""

    def __init__(self, fresh, length, heads=8, kv_heads=2, dim=128, dtype=torch.bfloat16, seed=17, out=None):
        torch.manual_seed(seed)
        rng = np.random.default_rng(seed)
        need = [-(-n // 16) for n in length]
        self.kc, self.vc = (torch.randn((sum(need) + 2, 16, kv_heads, dim), device="cuda").to(dtype) for _ in range(2))
        order, table, at = rng.permutation(sum(need) + 2), np.full((len(fresh), max(need + [1])), -1), 0
        for r, n in enumerate(need):
            table[r, :n] = order[at:at + n]
            at += n
        self.table, self.length, self.scale = _i32(table), _i32(length), dim ** -0.5
        self.q_start, self.max_q = _i32(np.concatenate([[0], np.cumsum(fresh)])), max(fresh)
        self.q = torch.randn((sum(fresh), heads, dim), device="cuda").to(dtype)
        self.out = torch.empty_like(self.q) if out is None else out(self.q)
        self.lse = torch.empty(self.q.shape[:2], device="cuda")
        self.clear()

    def clear(self):
        self.out.fill_(math.nan)
        self.lse.fill_(math.nan)

    def run(self, pp, kv, stream=None):
        pp.pp_paged_attention(kv, self.q, self.kc, self.vc, self.table, self.q_start, self.length, self.max_q, self.out,
                              self.scale, lse=self.lse, stream=stream)

    def check(self):
        rows = int(self.q_start[-1])
        want, lse, tol, lse_tol = ref.attention(self.q, self.kc, self.vc, self.table, self.q_start.tolist(),
                                                self.length.tolist(), self.scale, 0)
        assert ((self.out[:rows].double() - want[:rows]).abs() <= tol[:rows]).all()
        empty = lse[:rows] == -math.inf
        assert torch.equal(self.lse[:rows] == -math.inf, empty)
        assert ((self.lse[:rows].double() - lse[:rows]).abs() <= lse_tol[:rows])[~empty].all()
        assert self.out[rows:].isnan().all() and self.lse[rows:].isnan().all()


@pytest.mark.parametrize("fresh,length,then_start,then_length", [
    ([1, 1], [300, 77], [0, 1, 2], [299, 70]), ([4, 2], [300, 9000], [0, 3, 6], [20, 8000]),
    ([60, 140], [500, 300], [0, 100, 180], [100, 300]), ([300, 40], [900, 9000], [0, 1, 200], [30, 8999])])
def test_in_a_graph(pp, fresh, length, then_start, then_length):
    """Replayed with other lengths and queries than it was captured with."""
    step = _Step(fresh, length)
    with pp.KVCache.like(step.kc) as kv:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step.run(pp, kv)
        for change in range(2):
            step.clear()
            for _ in range(3):
                graph.replay()
            kv.sync()
            step.check()
            step.q_start.copy_(_i32(then_start))
            step.length.copy_(_i32(then_length))
            step.q.mul_(0.5)


@pytest.mark.parametrize("fresh", [[1, 1, 1], [3, 1, 4], [70, 1, 140]])
@pytest.mark.parametrize("dim,lead", [(128, 8), (64, 16), (72, 8)])
def test_in_a_wider_buffer(pp, fresh, dim, lead):
    buf = {}

    def out(q):
        buf["all"] = torch.full((q.shape[0], q.shape[1] * dim + 2 * lead), 3.0, dtype=q.dtype, device="cuda")
        return buf["all"][:, lead:-lead].unflatten(1, q.shape[1:])
    step = _Step(fresh, [f + 90 for f in fresh], heads=6, dim=dim, out=out)
    with pp.KVCache.like(step.kc) as kv:
        step.run(pp, kv)
        kv.sync()
    step.check()
    assert (buf["all"][:, :lead] == 3).all() and (buf["all"][:, -lead:] == 3).all()


@pytest.mark.parametrize("dim", [64, 128])
def test_in_many_pieces_by_turns(pp, dim):
    """One handle's calls, whose joins leave scratch and counters to the next."""
    whole = _Step([1], [40_000], dim=dim)
    steps = [whole]
    for fresh, length in (([40], [20_000]), ([30, 50], [5000, 9000]), ([4], [20_000]), ([90, 3, 200], [300, 6000, 8000])):
        s = _Step(fresh, length, dim=dim)
        s.kc, s.vc = whole.kc, whole.vc                     # the blocks of the largest
        steps.append(s)
    with pp.KVCache.like(whole.kc) as kv:
        for turn in range(4):
            for s in steps:
                s.clear()
                s.run(pp, kv)
        kv.sync()
    for s in steps:
        s.check()


def test_on_two_streams(pp):
    """Two handles' calls at the same time."""
    pairs = [[_Step(f, n, seed=s) for f, n in (([50], [11_000]), ([300], [10_000]), ([2], [11_200]))] for s in (1, 2)]
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    handles = [[pp.KVCache.like(s.kc) for s in steps] for steps in pairs]
    torch.cuda.synchronize()
    for turn in range(6):
        for steps, kvs, stream in zip(pairs, handles, streams):
            for s, kv in zip(steps, kvs):
                s.run(pp, kv, stream=stream)
    torch.cuda.synchronize()
    for steps, kvs in zip(pairs, handles):
        for s, kv in zip(steps, kvs):
            kv.sync()
            kv.close()
            s.check()


@pytest.mark.parametrize("fresh,length", [([1] * 9, [1, 2, 15, 16, 17, 64, 65, 128, 701]), ([3, 1, 65, 130], [3, 701, 129, 261]),
                                          ([40, 200, 3], [30, 50, 0]), ([4, 8, 3], [2, 1, 0]), ([1, 1], [20_000, 0])])
@pytest.mark.parametrize("heads,kv_heads,dim,dtype", [(7, 1, 128, torch.bfloat16), (4, 4, 64, torch.float16),
                                                      (16, 2, 80, torch.float16), (6, 3, 8, torch.bfloat16)])
def test_every_row_is_written(pp, fresh, length, heads, kv_heads, dim, dtype):
    step = _Step(fresh, length, heads, kv_heads, dim, dtype)
    with pp.KVCache.like(step.kc) as kv:
        step.run(pp, kv)
        kv.sync()
    step.check()
