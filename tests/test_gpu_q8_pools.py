"""The pools of an 8-bit cache for the page operations, and the descriptors of pools in C callers' memory."""
import ctypes

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rt():
    import torch
    from paper_2606_07665_b200 import build, runner
    build.build()
    torch.cuda.set_device(0)
    return runner


def codes(pages, ps, H, d):
    import torch
    return [torch.zeros(pages, ps, H, d, dtype=torch.int8, device="cuda") for _ in range(2)]


@pytest.mark.parametrize("pages", [1, 2, 5])
@pytest.mark.parametrize("H,ps,block", [(1, 16, 16), (3, 16, 16), (1, 48, 16), (2, 32, 16)])
def test_pools_of_empty_caches(rt, pages, H, ps, block):
    """Also of a single page, whose scales are no multiple of 16 bytes: forked into nothing, copied, compacted."""
    import torch
    cache = rt.Q8Cache.empty(pages, ps, H, 64, block)
    pools = cache.pools
    held = pools[2][0]
    assert held.shape[0] == pages and held.shape[1] % 4 == 0 and held.shape[1] - H * (ps // block) * 2 in range(4)
    assert held.data_ptr() == cache.scales.data_ptr()
    table, lens = torch.zeros(1, 4, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    refs = torch.zeros(pages, dtype=torch.int32, device="cuda")
    book = rt.CachePages(pools, table, lens, refs, page_size=ps)
    book.reserve(1)
    lens += 1
    book.copy(torch.tensor([[0, pages - 1]], dtype=torch.int32, device="cuda"))
    book.compact()
    torch.cuda.synchronize()
    assert int(book.status_flag) == 0 and refs.tolist() == [1] + [0] * (pages - 1)


@pytest.mark.parametrize("layers", [2, 3])
@pytest.mark.parametrize("H,ps,block", [(2, 32, 16), (4, 16, 16), (1, 64, 16)])
def test_scales_of_layers_side_by_side(rt, layers, H, ps, block):
    """Pages of one layer's scales with other layers' between them: calls take them, the page operations would move the others' too."""
    import torch
    every = torch.zeros(6, layers, H, ps // block, 2, device="cuda")
    for layer in range(layers):
        cache = rt.Q8Cache(*codes(6, ps, H, 64), every[:, layer])
        with pytest.raises(ValueError, match="scales"):
            cache.pools
        one = rt.Q8Cache(*codes(1, ps, H, 64), every[2:3, layer]).pools[2][0]      # of a single page nothing lies between
        assert one.shape == (1, H * (ps // block) * 2) and one.data_ptr() == every[2, layer].data_ptr()
    apart = torch.zeros(layers, 6, H, ps // block, 2, device="cuda")
    for layer in range(layers):
        assert len(rt.Q8Cache(*codes(6, ps, H, 64), apart[layer]).pools) == 3


def test_scales_without_room_behind_the_last_page(rt):
    import torch
    flat = torch.zeros(3 * 4 - 2, device="cuda")
    short = flat.as_strided((3, 1, 1, 2), (4, 2, 2, 1))
    with pytest.raises(ValueError, match="scales"):
        rt.Q8Cache(*codes(3, 16, 1, 64), short).pools
    room = torch.zeros(3 * 4, device="cuda").as_strided((3, 1, 1, 2), (4, 2, 2, 1))
    assert len(rt.Q8Cache(*codes(3, 16, 1, 64), room).pools) == 3


def test_pools_that_were_described_without_the_last_member(rt):
    """The int behind `segments` has never had a meaning for callers that copy by slots: whatever it holds, a fork copies the filled slots."""
    import torch
    from paper_2606_07665_b200 import binding as ac
    rng = np.random.default_rng(1)
    ps, pages = 16, 4
    for junk in (1, -1, 0x7FFFFFFF, 77):
        pool = torch.from_numpy(rng.integers(1, 100, (pages, ps, 64)).astype(np.uint8)).cuda()
        before = pool.clone()
        described = ac.page_pools([(pool, ps * 64, 1)])
        ctypes.memmove(ctypes.addressof(described) + 20, ctypes.byref(ctypes.c_int(junk)), 4)
        table = torch.tensor([[2, -1], [-1, -1]], dtype=torch.int32, device="cuda")
        lens = torch.tensor([5, -1], dtype=torch.int32, device="cuda")
        refs = torch.tensor([0, 0, 1, 0], dtype=torch.int32, device="cuda")
        pairs = torch.tensor([[0, 1]], dtype=torch.int32, device="cuda")
        room = torch.zeros(ac.ac_cache_workspace_bytes(2, pages, 1), dtype=torch.uint8, device="cuda")
        ac.ac_init(0)
        ac.ac_cache_fork(described, 1, table, 2, lens, refs, pairs, 1, 2, ps, pages, room, room.numel())
        torch.cuda.synchronize()
        want = before.clone()
        want[0, :5] = before[2, :5]
        assert table[1, 0] == 0 and torch.equal(pool, want), junk
