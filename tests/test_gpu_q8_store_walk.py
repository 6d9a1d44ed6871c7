"""The bulk store of the 8-bit cache where a CTA goes through several pieces: many ragged rows, against the rows stored one call each and
against the oracle."""
import numpy as np
import pytest

from oracle import q8_cache_oracle as Q
from tests.test_gpu_q8 import bits, dev, host

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rt():
    import torch
    from paper_2606_07665_b200 import build, runner
    build.build()
    torch.cuda.set_device(0)
    return runner


def rows_of(rng, T, block):
    """Lengths that add up to T: runs of empty and of very short rows, rows about as long as a block, long ones."""
    lens, left = [], T
    while left > 0:
        n = int(rng.choice([0, 0, 1, 2, 5, block - 1, block, block + 1, 3 * block + 7, int(rng.integers(1, 1000))]))
        lens.append(min(n, left))
        left -= lens[-1]
    return np.array(lens + [0, 0])


class Rows:
    """Ragged rows, some of them inactive, with a page that is none in the middle of some, starting anywhere in a block."""

    def __init__(self, seed, T, ps, block):
        rng = self.rng = np.random.default_rng(seed)
        lens = self.lens = rows_of(rng, T, block)
        B = self.B = len(lens)
        self.off = (3 + np.concatenate([[0], np.cumsum(lens)])).astype(np.int32)
        self.total = int(self.off[-1]) + 4
        self.start = (rng.integers(0, 3 * block, B) * (rng.random(B) < 0.6)).astype(np.int32)
        need = -(-(self.start + lens) // ps) + 1
        self.num_pages = int(need.sum()) + 2
        perm = rng.permutation(self.num_pages)
        self.table = np.full((B, int(need.max())), -7, dtype=np.int32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = perm[at:at + n]
            at += n
        self.bad = rng.random(B) < 0.1
        for b in np.flatnonzero(self.bad):
            self.table[b, (self.start[b] + lens[b] // 2) // ps] = rng.choice([-1, self.num_pages])
        self.start[rng.random(B) < 0.1] = -1


def filled(rt, rng, rows, ps, H, d, block, fmt):
    """A cache of random codes under random scales, the same from the same generator."""
    import torch
    cache = rt.Q8Cache.empty(rows.num_pages, ps, H, d, block, torch.int8 if fmt == Q.INT8 else torch.float8_e4m3fn)
    gen = torch.Generator(device="cuda").manual_seed(int(rng))
    for pool in (cache.k_codes, cache.v_codes):
        raw = torch.randint(0, 255, pool.shape, generator=gen, device="cuda", dtype=torch.uint8)
        raw[(raw & 0x7F) == 0x7F] = 0                               # no NaN of e4m3
        raw[raw == 0x80] = 0                                        # no -128 of int8
        pool.view(torch.uint8).copy_(raw)
    cache.scales.copy_(torch.ldexp(torch.ones_like(cache.scales), torch.randint(-9, 3, cache.scales.shape, generator=gen, device="cuda")))
    return cache


# (tokens, heads, head size, page, block): units of a whole block of 16 and of 12 of 48 tokens; of 64 and of 256 tokens, several
# rounds of four and of sixteen warps
SIZES = [(24_000, 4, 64, 16, 16), (30_000, 4, 128, 48, 48), (40_000, 8, 64, 64, 64), (42_000, 32, 64, 256, 256), (76_000, 1, 128, 32, 16)]


@pytest.mark.parametrize("T,H,d,ps,block", SIZES)
@pytest.mark.parametrize("fmt", [Q.INT8, Q.E4M3])
def test_one_call_is_its_rows(rt, T, H, d, ps, block, fmt):
    import torch
    from paper_2606_07665_b200 import binding as ac
    r = Rows(T + block, T, ps, block)
    gen = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn(r.total, H, d, generator=gen, device="cuda").bfloat16() for _ in range(2))
    k *= torch.pow(2.0, torch.randint(-6, 4, (r.total, H, 1), generator=gen, device="cuda")).bfloat16()      # scales that grow
    v[1000::997, 0, 3] = float("inf")
    one, rows = (filled(rt, 9, r, ps, H, d, block, fmt) for _ in range(2))
    untouched = [t.clone() for t in (one.k_codes.view(torch.uint8), one.scales)]
    table, start, off = dev(r.table), dev(r.start), dev(r.off)
    one.store(k, v, table, start, off)
    zero = torch.zeros(1, dtype=torch.int32, device="cuda")
    for b in range(r.B):
        lo, hi = int(r.off[b]), int(r.off[b + 1])
        if hi > lo:                                                 # from a view that begins with the row
            ends = torch.cat([zero, zero + (hi - lo)])
            rows.store(k[lo:hi], v[lo:hi], table[b:b + 1], start[b:b + 1], ends)
    torch.cuda.synchronize()
    assert int(one.status_flag) == int(rows.status_flag) == ac.AC_FLAG_PAGE_OOB
    assert torch.equal(one.scales.view(torch.int32), rows.scales.view(torch.int32))
    for a, b in ((one.k_codes, rows.k_codes), (one.v_codes, rows.v_codes)):
        differ = (a.view(torch.uint8) != b.view(torch.uint8)).flatten(1).any(1)
        assert not bool(differ.any()), int(differ.sum())
    assert not torch.equal(one.k_codes.view(torch.uint8), untouched[0]) and not torch.equal(one.scales, untouched[1])


@pytest.mark.parametrize("T,H,d,ps,block", [(24_000, 4, 64, 16, 16), (20_000, 4, 64, 48, 48), (20_000, 4, 64, 256, 256)])
@pytest.mark.parametrize("fmt", [Q.INT8, Q.E4M3])
def test_rows_are_the_oracle_s(rt, T, H, d, ps, block, fmt):
    """A hundred rows of such a call, and every page that no row of it holds."""
    import torch
    r = Rows(T + 7, T, ps, block)
    k, v = bits(r.rng, r.total, H, d, scale=0.5), bits(r.rng, r.total, H, d, scale=3.0)
    cache = filled(rt, 11, r, ps, H, d, block, fmt)
    want = Q.Cache(host(cache.k_codes).copy(), host(cache.v_codes).copy(), host(cache.scales).copy(), fmt)
    cache.store(dev(k), dev(v), dev(r.table), dev(r.start), dev(r.off))
    torch.cuda.synchronize()
    got = [host(cache.k_codes), host(cache.v_codes)], host(cache.scales)
    held = np.unique(r.table[(r.table >= 0) & (r.table < r.num_pages)])
    free = np.setdiff1d(np.arange(r.num_pages), held)
    good = np.flatnonzero((r.lens > 0) & (r.start >= 0) & ~r.bad)
    still = np.flatnonzero((r.lens == 0) | (r.start < 0))
    checked = 0
    for b in np.concatenate([r.rng.choice(good, min(100, len(good)), replace=False), still[:50]]):
        pages = r.table[b][(r.table[b] >= 0) & (r.table[b] < r.num_pages)]
        if b in good:
            for side, x in enumerate((k, v)):
                want.store(x[r.off[b]:r.off[b + 1]], side, r.table[b], int(r.start[b]))
            checked += int(r.lens[b])
        assert np.array_equal(got[1][pages], want.scales[pages]), b
        for side in range(2):
            assert np.array_equal(got[0][side][pages], want.pools[side][pages]), (b, side)
    for side in range(2):
        assert np.array_equal(got[0][side][free], want.pools[side][free])
    assert checked > 1000
