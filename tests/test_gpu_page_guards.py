"""Page operations and bulk copies on lists that break their rules: everything stays inside the tables and the pools."""
import numpy as np
import pytest

from tests.test_gpu_cache_pages import Both, i32
from tests.test_gpu_q4 import bits, dev, host

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rt():
    import torch
    from paper_2606_07665_b200 import build, runner
    build.build()
    torch.cuda.set_device(0)
    return runner


def test_fork_goes_by_the_lengths_before_the_call(rt):
    """A row that is a child and a parent of one call: its child gets the length that the row had, however the two forks
    come to run, and nothing is written past the child's table row (the last one) when the row itself becomes longer."""
    import torch
    width, ps, rows = 8, 16, 40
    b = Both(rt, 80, [width * ps], ps, 400, width, rows)
    guarded = torch.full((rows + 1, width), -9, dtype=torch.int32, device="cuda")
    guarded[:rows] = b.h.block_table
    lens = b.h.context_lens
    mid = list(range(1, rows // 2))
    last = list(range(rows // 2, rows // 2 + len(mid)))
    at = 300
    for r in mid:                                          # used rows of 17 tokens, about to be overwritten
        guarded[r, :2] = i32([at, at + 1])
        b.h.ref_counts[at:at + 2] = 1
        lens[r] = 17
        at += 2
    h = rt.CachePages([b.t[0]], guarded[:rows], lens, b.h.ref_counts, ps)
    pairs = [(0, r) for r in mid] + list(zip(mid, last))
    h.fork(i32(pairs))
    torch.cuda.synchronize()
    got = lens.cpu().numpy()
    assert (got[last] == 17).all() and (got[mid] == width * ps).all()
    assert bool((guarded[rows] == -9).all())
    assert int(h.status_flag) == 0


@pytest.mark.parametrize("d,group,heads", [(128, 64, 8), (64, 32, 3)])
@pytest.mark.parametrize("first", [1, 5, 40, 400])
def test_bulk_tokens_before_the_first_row_belong_to_no_row(rt, d, group, heads, first):
    import torch
    rng = np.random.default_rng(81)
    B, ps, each = 3, 16, 30
    total = first + B * each
    cache = rt.Q4Cache.empty(B * 2 + 1, ps, heads, d, group)
    table = i32([[1, 2], [3, 4], [5, 6]])                  # page 0 belongs to nobody, and nothing lies in front of it
    before = [x.clone() for x in (cache.k_codes, cache.v_codes, cache.params)]
    k, v = dev(bits(rng, total, heads, d)), dev(bits(rng, total, heads, d))
    off, start = i32([first + each * b for b in range(B + 1)]), i32([0, 2, 1])
    cache.store(k, v, table, start, off)
    kb, vb = cache.load(table, start, off, total)
    torch.cuda.synchronize()
    assert int(cache.status_flag) == 0
    for x, y in zip(before, (cache.k_codes, cache.v_codes, cache.params)):
        assert torch.equal(x[0], y[0])
    for got, x in ((kb, k), (vb, v)):
        assert not host(got[:first]).any()                 # +0, not what the memory held
        alone = rt.Q4Cache.empty(B * 2 + 1, ps, heads, d, group)
        alone.store(x[first:], x[first:], table, start, off - first)
        want, _ = alone.load(table, start, off - first, total - first)
        assert torch.equal(got[first:], want)
