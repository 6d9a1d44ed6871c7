"""Page operations and bulk copies recorded into one graph and replayed on a state that goes on from replay to replay."""
import numpy as np
import pytest

from oracle import q4_cache_oracle as Q
from tests.test_gpu_cache_pages import Both, i32
from tests.test_gpu_pages_large import State, pick
from tests.test_gpu_q4 import bits, dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rt():
    import torch
    from paper_2606_07665_b200 import build, runner
    build.build()
    torch.cuda.set_device(0)
    return runner


@pytest.mark.parametrize("large", [False, True])
def test_page_operations_replayed(rt, large):
    import torch
    if large:                                              # several chunks, so that compaction has all of its launches
        s = State(rt, 120, [1 + i % 90 for i in range(300)] + [-1] * 40, pick(121, 20000, 2000), 20000, 14, n_pools=9)
        rows, alive = 340, 300
    else:
        s = Both(rt, 122, [40, 16, 0, 33, 1, 15], 16, 200, 14, 9)
        rows, alive = 9, 6
    pairs = [(i % alive, alive + i) for i in range(rows - alive)]
    gone = [c for _, c in pairs]
    pairs_d, gone_d, grow = i32(pairs), i32(gone), i32([1] * alive + [0] * (rows - alive))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.h.reserve(1)
        s.h.context_lens.add_(grow)
        s.h.fork(pairs_d)
        s.h.compact()
        s.h.release(gone_d)
        s.h.reserve(40)
        s.h.trim()
        s.h.compact()
    for _ in range(20):
        graph.replay()
        s.o.reserve(1)
        s.o.lens[:alive] += 1
        s.o.fork(pairs)
        s.o.compact()
        s.o.release(gone)
        s.o.reserve(40)                                    # leaves its entries in the table
        s.o.refs[:] = 0
        for r, n in enumerate(s.o.lens):
            for i in range(s.o.pages(max(int(n), 0))):
                s.o.refs[s.o.table[r, i]] += 1
        s.o.compact()
    s.same()


def test_store_and_load_replayed(rt):
    import torch
    rng = np.random.default_rng(123)
    heads, d, group, ps, T = 3, 128, 32, 16, 200
    cache = rt.Q4Cache.empty(40, ps, heads, d, group)
    table, start, off = i32(rng.permutation(40)[:30].reshape(2, 15).tolist()), i32([0, 0]), i32([0, 0, 0])
    k, v, kb, vb = (dev(np.zeros((T, heads, d), np.uint16)) for _ in range(4))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.store(k, v, table, start, off)
        cache.load(table, start, off, k_out=kb, v_out=vb)
    for n0, n1, s0, s1 in ((100, 100, 0, 0), (0, 200, 5, 40), (200, 0, 7, -1), (30, 1, -1, 239), (120, 80, 0, 3)):
        x = [bits(rng, T, heads, d) for _ in range(2)]
        k.copy_(dev(x[0])), v.copy_(dev(x[1]))
        start.copy_(i32([s0, s1])), off.copy_(i32([0, n0, n0 + n1]))
        graph.replay()
        torch.cuda.synchronize()
        for src, got in zip(x, (kb, vb)):
            codes, s, m = Q.quantise(src, group)
            want = Q.values(Q.pack(codes), s, m)[0]
            lost = np.ones(T, dtype=bool)                  # tokens of no row, or of an inactive one
            lost[:n0] = s0 < 0
            lost[n0:n0 + n1] = s1 < 0
            want[lost] = 0.0
            back = got.view(torch.bfloat16).double().cpu().numpy()
            assert (np.abs(back - want) <= 2.0**-8 * (1 + 2.0**-8) * np.abs(want)).all()
    assert int(cache.status_flag) == 0
