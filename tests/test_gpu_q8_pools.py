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
