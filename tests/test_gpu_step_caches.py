"""Which caches the decode steps take."""
import pytest

from tests.test_gpu_q4 import Case, bits, dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rt():
    import torch
    from paper_2606_07665_b200 import build, runner
    build.build()
    torch.cuda.set_device(0)
    return runner


class Described:
    """A cache of a caller's own class: the library's descriptor, and what it says."""

    def __init__(self, cache):
        self.device, self.struct, self._held = cache.device, cache.struct, cache
        self.num_pages, self.page_size, self.Hkv, self.d = cache.num_pages, cache.page_size, cache.Hkv, cache.d

    def _buffers(self):
        return self._held._buffers()


def test_caches_of_other_classes(rt):
    import torch
    c = Case(rt, 100, [100, 20], 4, 2, 64, 16, 32)
    cache = c.upload(rt)
    q = dev(bits(c.rng, 2, 4, 64))
    outs = [rt.Q4DecodeStep(x, dev(c.table), dev(c.lens), 4, lens_host=c.lens).attention(q) for x in (cache, Described(cache))]
    assert torch.equal(*outs)
    eight = rt.Q8Cache.empty(c.num_pages, 16, 2, 64)
    outs = [rt.Q8DecodeStep(x, dev(c.table), dev(c.lens), 4, lens_host=c.lens).attention(q) for x in (eight, Described(eight))]
    assert torch.equal(*outs)


def test_caches_of_the_other_format(rt):
    import torch
    table, lens = torch.zeros(1, 4, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    four, eight = rt.Q4Cache.empty(4, 32, 2, 64), rt.Q8Cache.empty(4, 32, 2, 64)
    for kind, wrong in ((rt.Q4DecodeStep, eight), (rt.Q8DecodeStep, four), (rt.Q4DecodeStep, Described(eight)), (rt.Q8DecodeStep, Described(four)),
                        (rt.Q8DecodeStep, None), (rt.Q4DecodeStep, four.k_codes)):
        with pytest.raises(TypeError, match="cache"):
            kind(wrong, table, lens, 4)
