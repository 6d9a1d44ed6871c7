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
