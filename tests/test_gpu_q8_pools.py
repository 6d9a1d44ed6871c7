"""The pools of an 8-bit cache for the page operations."""
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
