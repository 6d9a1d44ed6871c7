"""Page operations on the GPU against plain Python: tables, lengths, counts and pool bytes are compared exactly."""
import numpy as np
import pytest

from oracle import q4_cache_oracle as Q

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rt():
    import torch
    from paper_2606_07665_b200 import build, runner
    build.build()
    torch.cuda.set_device(0)
    return runner


class Both:
    """The same state in the oracle and on the GPU."""

    def __init__(self, rt, seed, lens, ps, num_pages, width, rows=None, shared=(), slot_bytes=48, heads=3):
        import torch
        rng = np.random.default_rng(seed)
        rows = len(lens) if rows is None else rows
        full = np.full(rows, -1, dtype=np.int32)
        full[:len(lens)] = lens
        table = rng.integers(0, num_pages, (rows, width)).astype(np.int32)       # entries past a row's pages hold anything
        refs = np.zeros(num_pages, dtype=np.int32)
        perm, at = rng.permutation(num_pages), 0
        for r, n in enumerate(full):
            k = -(-max(int(n), 0) // ps)
            table[r, :k] = perm[at:at + k]
            at += k
            refs[table[r, :k]] += 1
        for a, b in shared:                                                        # row b shares row a's full pages
            k = int(full[a]) // ps
            table[b, :k] = table[a, :k]
            full[b] = k * ps
            refs[table[a, :k]] += 1
        pools = [(rng.integers(0, 256, (num_pages, ps, heads, slot_bytes // heads)).astype(np.uint8), 1),     # token-major
                 (rng.integers(0, 256, (num_pages, heads, ps, 8)).astype(np.uint8), 2),                          # head-major, 8 bytes a slot
                 (rng.integers(0, 256, (num_pages, ps, 8, 512)).astype(np.uint8), 1)]                             # pages of several pieces
        self.o = Q.Pages(table, full, refs, ps, pools)
        up = lambda x: torch.from_numpy(x.copy()).cuda()                                                          # noqa: E731
        self.t = [up(p) for p, _ in pools]
        self.h = rt.CachePages([self.t[0], (self.t[1], heads), self.t[2]], up(table), up(full), up(refs), ps)

    def same(self, flags=0, pools=True):
        import torch
        torch.cuda.synchronize()
        assert int(self.h.status_flag) == flags
        assert np.array_equal(self.h.context_lens.cpu().numpy(), self.o.lens), "lengths"
        assert np.array_equal(self.h.ref_counts.cpu().numpy(), self.o.refs), "counts"
        assert np.array_equal(self.h.block_table.cpu().numpy(), self.o.table), "table"
        for i, (p, _) in enumerate(self.o.pools if pools else []):
            assert np.array_equal(self.t[i].cpu().numpy(), p), f"pool {i}"


def i32(x):
    import torch
    return torch.tensor(x, dtype=torch.int32, device="cuda")


CASES = [([40, 16, 0, 33, 1, 15], 16, 64, 8, 12), ([100], 48, 20, 4, 3), ([5, 700, -1, 64], 32, 1000, 30, 9), ([300] * 20, 16, 20000, 25, 60)]


@pytest.mark.parametrize("lens,ps,num_pages,width,rows", CASES)
@pytest.mark.parametrize("new_tokens", [1, 16, 33])
def test_reserve(rt, lens, ps, num_pages, width, rows, new_tokens):
    b = Both(rt, 1, lens, ps, num_pages, width, rows)
    b.h.reserve(new_tokens)
    b.o.reserve(new_tokens)
    b.same()


def test_reserve_runs_out_and_past_the_table(rt):
    from paper_2606_07665_b200 import binding as ac
    b = Both(rt, 2, [32, 16, 48, 31, 5], 16, 12, 8)                # 9 pages held, 3 free
    b.h.reserve(17)                                                  # rows need 2, 2, 2, 1, 1
    b.o.reserve(17)
    b.same(ac.AC_FLAG_POOL_EXHAUSTED)
    b = Both(rt, 3, [128, 16], 16, 40, 8)
    b.h.reserve(1)
    b.o.reserve(1)
    b.same(ac.AC_FLAG_POSITION_OOB)
    b = Both(rt, 3, [16], 16, 1, 4)                                  # nothing free at all
    b.h.reserve(1)
    b.o.reserve(1)
    b.same(ac.AC_FLAG_POOL_EXHAUSTED)


@pytest.mark.parametrize("lens,ps,num_pages,width,rows", CASES)
def test_fork_then_release(rt, lens, ps, num_pages, width, rows):
    b = Both(rt, 4, lens, ps, num_pages, width, rows)
    free_rows = list(range(len(lens), rows))
    pairs = [(i % len(lens), c) for i, c in enumerate(free_rows)]
    pairs = [p for p in pairs]
    b.h.fork(i32(pairs))
    b.o.fork(pairs)
    b.same()
    b.h.release(i32(free_rows[::2] + [0]))
    b.o.release(free_rows[::2] + [0])
    b.same()


def test_fork_exhausted_unused_and_out_of_range(rt):
    from paper_2606_07665_b200 import binding as ac
    b = Both(rt, 5, [20, 32, -1], 16, 6, 4, rows=9)                # 4 pages held, 2 free
    pairs = [(0, 3), (1, 4), (2, 5), (0, 6), (0, 7)]                # the last one finds no page
    b.h.fork(i32(pairs))
    b.o.fork(pairs)
    b.same(ac.AC_FLAG_POOL_EXHAUSTED)
    assert list(b.o.lens[3:8]) == [20, 32, -1, 20, -1]
    b.h.fork(i32([(0, 9), (-1, 8), (12, 8)]))                        # rows that are not there: nothing changes
    b.same(ac.AC_FLAG_POOL_EXHAUSTED | ac.AC_FLAG_ROW_OOB)


def test_fork_of_nothing(rt):
    import torch
    b = Both(rt, 5, [20], 16, 6, 4, rows=3)
    b.h.fork(torch.zeros(0, 2, dtype=torch.int32, device="cuda"))
    b.h.release(torch.zeros(0, dtype=torch.int32, device="cuda"))
    b.h.copy(torch.zeros(0, 2, dtype=torch.int32, device="cuda"))
    b.h.reserve(0)
    b.same()
    with pytest.raises(ValueError):
        b.h.fork(i32([(0, 1)] * 4))


def test_release_twice(rt):
    from paper_2606_07665_b200 import binding as ac
    b = Both(rt, 6, [40, 40, 40], 16, 30, 4, rows=5, shared=[(0, 3)])
    b.h.release(i32([1, 3, 1, 4]))                                   # listed twice; unused: no-ops
    b.o.release([1, 3])
    b.same()
    b.h.ref_counts[b.o.table[2, 1]] = 0                              # a page that was never counted
    b.o.refs[b.o.table[2, 1]] = 1
    b.h.release(i32([2, 99]))
    b.o.release([2])
    b.same(ac.AC_FLAG_REF_COUNT | ac.AC_FLAG_ROW_OOB)


@pytest.mark.parametrize("lens,ps,num_pages,width,rows,shared", [
    ([40, 16, 0, 33, 1, 15], 16, 64, 8, 12, [(0, 6)]), ([100], 48, 20, 4, 3, []), ([], 16, 37, 4, 3, []), ([64] * 10, 16, 40, 4, 10, []),
    ([5, 700, -1, 64], 32, 1001, 30, 9, [(1, 4), (1, 5)]), ([300] * 20, 16, 40000, 25, 60, [(3, 22)])])
@pytest.mark.parametrize("in_place", [True, False])
def test_compact(rt, lens, ps, num_pages, width, rows, shared, in_place):
    import torch
    b = Both(rt, 7, lens, ps, num_pages, width, rows, shared)
    before = [x.clone() for x in (b.h.block_table, b.h.ref_counts)]
    live = i32([-1])
    out = (None, None) if in_place else (torch.full_like(before[0], -5), torch.full_like(before[1], -5))
    b.h.compact(*out, live_out=live)
    torch.cuda.synchronize()
    if not in_place:
        assert torch.equal(b.h.block_table, before[0]) and torch.equal(b.h.ref_counts, before[1])
        b.h.block_table.copy_(out[0])
        b.h.ref_counts.copy_(out[1])
    assert int(live) == b.o.compact()
    b.same()
    b.h.compact()                                                    # compact already: nothing moves
    b.same()


def test_copy_pages(rt):
    from paper_2606_07665_b200 import binding as ac
    b = Both(rt, 8, [40], 16, 300, 4)
    pairs = [(i, 299 - i) for i in range(100)] + [(150, 150)]
    b.h.copy(i32(pairs + [(5, 300), (-1, 7)]))
    for p, _ in b.o.pools:
        for s, d in pairs:
            p[d] = p[s]
    b.same(ac.AC_FLAG_PAGE_OOB)


def test_beam_search_over_the_4_bit_cache(rt):
    # the operators together: prompts stored, rows grown, forked, dropped and compacted between attention steps; a row's
    # attention does not change when its pages move, and a child attends over its parent's tokens
    import torch
    rng = np.random.default_rng(9)
    Hq, Hkv, d, ps, rows, num_pages, width = 8, 2, 64, 16, 8, 120, 10
    cache = rt.Q4Cache.empty(num_pages, ps, Hkv, d, 32, layout="head_major")
    table, lens, refs = i32(np.zeros((rows, width)).tolist()), i32([0, 0, 0] + [-1] * 5), i32([0] * num_pages)
    pages = rt.CachePages(cache.pools, table, lens, refs, ps)
    n = [37, 80, 5]
    pages.reserve(85)
    lens[:3] = i32(n)
    off = i32([0, 37, 117, 122] + [122] * (rows - 3))
    kv = [torch.randn(122, Hkv, d, device="cuda").to(torch.bfloat16) for _ in range(2)]
    cache.store(*kv, table, i32([0] * rows), off)
    # the reservation was for 85 tokens: hand back what the prompts did not take
    held = torch.zeros_like(refs)
    for r in range(3):
        held[table[r, :-(-n[r] // ps)].long()] = 1
    refs.copy_(held)
    cos = torch.ones(200, d // 2, device="cuda")
    step = rt.Q4DecodeStep(cache, table, lens, Hq, max_context_len=width * ps, rope_cos=cos, rope_sin=torch.zeros_like(cos))
    q = torch.randn(rows, Hq, d, device="cuda").to(torch.bfloat16)

    def attend():
        step.new_tokens = 0
        step._marshal()
        return step.attention(q).clone()

    pages.fork(i32([(0, 3), (0, 4), (1, 5), (1, 6)]))
    q[3:7] = q[torch.tensor([0, 0, 1, 1], device="cuda")]
    a = attend()
    assert torch.equal(a[3], a[0]) and torch.equal(a[4], a[0]) and torch.equal(a[5], a[1]) and torch.equal(a[6], a[1])
    assert not a[7].any()                                              # unused
    for i in range(20):                                                # every row grows on its own pages
        pages.reserve(1)
        new = [torch.randn(rows, h, d, device="cuda").to(torch.bfloat16) for h in (Hq, Hkv, Hkv)]
        step.new_tokens = 1
        step._marshal()
        step.step(*new)
        lens.add_((lens >= 0).int())
        if i == 10:
            pages.release(i32([0, 5]))
            before = attend()
            pages.compact()
            assert torch.equal(attend(), before)
            live = int((refs > 0).sum())
            assert bool((refs[:live] > 0).all()) and not bool(refs[live:].any())
    torch.cuda.synchronize()
    assert int(pages.status_flag) == 0 and int(step.status_flag) == 0
    # parent and children share the prompt's full pages and nothing else
    t = table.cpu().numpy()
    assert (t[1, :5] == t[6, :5]).all() and t[1, 5] != t[6, 5] and (t[3, :2] == t[4, :2]).all() and t[3, 2] != t[4, 2]
    pages.release(i32(list(range(rows))))
    assert not bool(refs.any())
