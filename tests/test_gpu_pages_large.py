"""Page operations past the sizes of one step of their kernels: pools of several chunks of 4096 pages and of several steps of
16384, more rows and forks than a CTA has threads, and as many pools as a call takes."""
import numpy as np
import pytest

from oracle import q4_cache_oracle as Q
from tests.test_gpu_cache_pages import i32

pytestmark = pytest.mark.gpu

PS = 16


@pytest.fixture(scope="module")
def rt():
    import torch
    from paper_2606_07665_b200 import build, runner
    build.build()
    torch.cuda.set_device(0)
    return runner


class State:
    """The same state in the oracle and on the GPU; `occupied` are the pages that count as held, rows take theirs from them."""

    def __init__(self, rt, seed, lens, occupied, num_pages, width, n_pools=1):
        import torch
        rng = np.random.default_rng(seed)
        lens = np.asarray(lens, dtype=np.int32)
        table = rng.integers(0, num_pages, (len(lens), width)).astype(np.int32)
        refs = np.zeros(num_pages, dtype=np.int32)
        refs[occupied] = 1
        mine, at = rng.permutation(occupied), 0
        for r, n in enumerate(lens):
            k = -(-max(int(n), 0) // PS)
            table[r, :k] = mine[at:at + k]
            at += k
        assert at <= len(mine)
        # pools of 32 bytes a page (two bytes a slot); every third with two segments
        pools = [(rng.integers(0, 256, (num_pages, PS, 2) if i % 3 else (num_pages, 2, PS, 1)).astype(np.uint8), 1 if i % 3 else 2) for i in range(n_pools)]
        self.o = Q.Pages(table, lens, refs, PS, pools)
        up = lambda x: torch.from_numpy(x.copy()).cuda()                       # noqa: E731
        self.t = [up(p) for p, _ in pools]
        self.h = rt.CachePages([(t, axis) for t, (_, axis) in zip(self.t, pools)], up(table), up(lens), up(refs), PS)

    def same(self, flags=0):
        import torch
        torch.cuda.synchronize()
        assert int(self.h.status_flag) == flags
        assert np.array_equal(self.h.context_lens.cpu().numpy(), self.o.lens), "lengths"
        assert np.array_equal(self.h.ref_counts.cpu().numpy(), self.o.refs), "counts"
        assert np.array_equal(self.h.block_table.cpu().numpy(), self.o.table), "table"
        for i, (p, _) in enumerate(self.o.pools):
            assert np.array_equal(self.t[i].cpu().numpy(), p), f"pool {i}"


def pick(seed, num_pages, n, low=0):
    return np.sort(np.random.default_rng(seed).permutation(np.arange(low, num_pages))[:n])


@pytest.mark.parametrize("num_pages,live", [
    (4096, 4096), (4096, 4095), (4095, 4095), (8192, 4096), (8192, 4097), (8192, 8192), (8193, 8192), (8193, 1), (20000, 10000), (20001, 16384),
    (40000, 12289), (70000, 69999), (12288, 0)])
@pytest.mark.parametrize("where", ["scattered", "behind", "in front"])
def test_compact_several_chunks(rt, num_pages, live, where):
    occupied = {"scattered": pick(1, num_pages, live), "behind": np.arange(num_pages - live, num_pages), "in front": np.arange(live)}[where]
    lens, left = [], live
    rng = np.random.default_rng(2)
    while left > 0 and len(lens) < 400:
        k = min(left, int(rng.integers(1, 60)))
        lens.append(k * PS - int(rng.integers(0, PS)))
        left -= k
    s = State(rt, 3, lens + [-1], occupied, num_pages, 60)
    n = i32([-1])
    s.h.compact(live_out=n)
    assert int(n) == s.o.compact() == live
    s.same()


# free pages in the first step of 16384, in the second, in the third
@pytest.mark.parametrize("free", [(5, 7, 400), (0, 0, 400), (0, 400, 0), (1, 0, 399), (150, 150, 10), (100, 95, 5), (16384, 0, 0)])
def test_reserve_and_fork_several_steps(rt, free):
    from paper_2606_07665_b200 import binding as ac
    num_pages = 2 * 16384 + 5000
    open_ = np.concatenate([pick(4 + i, min(num_pages, (i + 1) * 16384), n, i * 16384) for i, n in enumerate(free)])
    occupied = np.setdiff1d(np.arange(num_pages), open_)
    s = State(rt, 5, [33 + i for i in range(100)] + [-1] * 120, occupied, num_pages, 12, n_pools=2)
    s.h.reserve(20)
    s.o.reserve(20)
    s.same(0)
    pairs = [(i % 100, 100 + i) for i in range(120)]
    s.h.fork(i32(pairs))
    s.o.fork(pairs)
    s.same(ac.AC_FLAG_POOL_EXHAUSTED if any(s.o.lens[100:] < 0) else 0)


@pytest.mark.parametrize("rows,forks", [(1025, 1024), (3000, 1025), (2048, 2500)])
def test_more_rows_and_forks_than_threads(rt, rows, forks):
    lens = [1 + i % 40 for i in range(rows)] + [-1] * forks
    need = sum(-(-max(n, 0) // PS) for n in lens)
    num_pages = 3 * need + 2 * forks
    s = State(rt, 6, lens, pick(7, num_pages, need), num_pages, 4, n_pools=2)
    s.h.reserve(17)
    s.o.reserve(17)
    s.same()
    s.h.trim()
    s.o.refs[:] = 0
    for r in range(rows):
        for i in range(s.o.pages(lens[r])):
            s.o.refs[s.o.table[r, i]] += 1
    s.same()
    pairs = [(int(p), rows + i) for i, p in enumerate(np.random.default_rng(8).integers(0, rows, forks))]
    s.h.fork(i32(pairs))
    s.o.fork(pairs)
    s.same()
    gone = list(range(0, rows + forks, 2))
    s.h.release(i32(gone))
    s.o.release(gone)
    s.same()
    s.h.compact()
    s.o.compact()
    s.same()


@pytest.mark.parametrize("n_pools", [8, 9, 96, 128])
def test_many_pools(rt, n_pools):
    s = State(rt, 9, [40, 16, 33, 7, -1, -1, -1], pick(10, 300, 9), 300, 5, n_pools=n_pools)
    pairs = [(0, 4), (2, 5), (3, 6)]
    s.h.fork(i32(pairs))
    s.o.fork(pairs)
    s.same()
    held = np.unique(s.o.table[0, :3])
    copies = [(int(a), 290 + i) for i, a in enumerate(held)]
    s.h.copy(i32(copies))
    for p, _ in s.o.pools:
        for a, b in copies:
            p[b] = p[a]
    s.same()
    s.h.release(i32([0]))
    s.o.release([0])
    s.h.compact()
    s.o.compact()
    s.same()


def test_one_pool_too_many(rt):
    from paper_2606_07665_b200 import binding as ac
    s = State(rt, 11, [40], pick(12, 30, 3), 30, 5, n_pools=129)
    with pytest.raises(ac.AcError) as e:
        s.h.compact()
    assert e.value.status == 3
    s.same()
