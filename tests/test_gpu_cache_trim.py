"""Pages that were reserved and not used come back, and no others."""
import numpy as np
import pytest

from tests.test_gpu_cache_pages import Both, i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rt():
    import torch
    from paper_2606_07665_b200 import build, runner
    build.build()
    torch.cuda.set_device(0)
    return runner


def held(b):
    """The counts that the oracle's rows stand for."""
    refs = np.zeros_like(b.o.refs)
    for r, n in enumerate(b.o.lens):
        for i in range(b.o.pages(max(int(n), 0))):
            refs[b.o.table[r, i]] += 1
    return refs


def trimmed(b, flags=0):
    b.h.trim()
    b.o.refs[:] = held(b)
    b.same(flags)


CASES = [([40, 16, 0, 33, 1, 15], 16, 64, 8, 12, [(0, 6)]), ([100], 48, 20, 4, 3, []), ([], 16, 37, 4, 3, []), ([5, 700, -1, 64], 32, 1001, 30, 9, [(1, 4), (1, 5)]),
         ([300] * 20, 16, 2000, 25, 60, [(3, 22)]), ([15] * 1500, 16, 3000, 2, 1500, [])]


@pytest.mark.parametrize("lens,ps,num_pages,width,rows,shared", CASES)
def test_released_without_having_grown(rt, lens, ps, num_pages, width, rows, shared):
    b = Both(rt, 90, lens, ps, num_pages, width, rows, shared)
    trimmed(b)                                             # nothing reserved: nothing changes
    b.h.reserve(ps + 1)
    b.o.reserve(ps + 1)
    b.h.release(i32(list(range(rows))))
    b.o.release(range(rows))
    trimmed(b)
    assert not b.o.refs.any()


@pytest.mark.parametrize("lens,ps,num_pages,width,rows,shared", CASES)
def test_grown_by_less_than_was_reserved(rt, lens, ps, num_pages, width, rows, shared):
    from paper_2606_07665_b200 import binding as ac
    b = Both(rt, 91, lens, ps, num_pages, width, rows, shared)
    rng = np.random.default_rng(92)
    flags = 0
    for _ in range(4):
        if any(n >= 0 and b.o.pages(n + 2 * ps) > width for n in b.o.lens):
            flags = ac.AC_FLAG_POSITION_OOB                 # reserve says so, and gives that row nothing
        b.h.reserve(2 * ps)
        b.o.reserve(2 * ps)
        room = np.array([0 if n < 0 or b.o.pages(n + 2 * ps) > width else 2 * ps for n in b.o.lens])
        b.o.lens += (rng.random(rows) * (room + 1)).astype(np.int32)       # some grow by nothing, some by all of it
        b.h.context_lens.copy_(i32(b.o.lens.tolist()))
        trimmed(b, flags)
    assert b.o.refs.sum() == sum(b.o.pages(max(int(n), 0)) for n in b.o.lens)


def test_pages_of_ragged_prompts_then_compaction(rt):
    # one count for all rows when they are admitted, what the short ones did not need back, then the pool made dense
    b = Both(rt, 93, [0, 0, 0, 0], 16, 200, 10, 6)
    b.h.reserve(150)
    b.o.reserve(150)
    b.o.lens[:4] = [37, 150, 5, 0]
    b.h.context_lens.copy_(i32(b.o.lens.tolist()))
    trimmed(b)
    b.h.compact()
    assert b.o.compact() == 3 + 10 + 1
    b.same()


def test_trim_of_rows_that_do_not_fit(rt):
    from paper_2606_07665_b200 import binding as ac
    b = Both(rt, 94, [40, 16], 16, 30, 4, 3)
    b.h.context_lens[1] = 65                               # longer than its table row: as far as that goes
    b.h.block_table[0, 1] = 30
    b.h.block_table[1] = i32([3, 3, 4, 5])
    b.h.trim()
    want = np.zeros(30, dtype=np.int32)
    for p in (b.o.table[0, 0], b.o.table[0, 2], 3, 3, 4, 5):
        want[p] += 1
    assert np.array_equal(b.h.ref_counts.cpu().numpy(), want)
    assert int(b.h.status_flag) == ac.AC_FLAG_POSITION_OOB | ac.AC_FLAG_PAGE_OOB
