"""What the objects over the caller's tensors refuse before anything is launched."""
import numpy as np
import pytest

from paper_2606_07665_b200 import workloads as W
from tests.test_gpu_q4 import Case, bits, dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rt():
    import torch
    from paper_2606_07665_b200 import build, runner
    build.build()
    torch.cuda.set_device(0)
    return runner


@pytest.fixture(scope="module")
def case(rt):
    c = Case(rt, 100, [10, 20], 4, 2, 64, 16, 32)
    cache = c.upload(rt)
    cos, sin = (dev(x) for x in W.rope_table(64, 64, 10000.0))
    return c, cache, cos, sin


@pytest.mark.parametrize("which", ["q_norm_weight", "k_norm_weight"])
def test_norm_weights(rt, case, which):
    import torch
    c, cache, cos, sin = case
    good = torch.ones(64, dtype=torch.bfloat16, device="cuda")

    def make(weight):
        return rt.Q4DecodeStep(cache, dev(c.table), dev(c.lens), 4, lens_host=c.lens, rope_cos=cos, rope_sin=sin,
                               rope_variants={which: weight, "norm_eps": 1e-5})

    for bad in (good.cpu(), good.float(), good[:32], torch.ones(128, dtype=torch.bfloat16, device="cuda")[::2], good.reshape(1, 64)):
        with pytest.raises(ValueError, match=which):
            make(bad)
    with pytest.raises(TypeError, match=which):
        make(good.data_ptr())
    make(good)
    make(good.view(torch.int16))


def test_rope_tables_come_in_pairs(rt, case):
    c, cache, cos, sin = case

    def make(a, b, **variants):
        return rt.Q4DecodeStep(cache, dev(c.table), dev(c.lens), 4, lens_host=c.lens, rope_cos=a, rope_sin=b, rope_variants=variants)

    for a, b in ((cos, None), (None, sin), (cos, sin[:32]), (cos, sin.cpu()), (cos, sin.double()), (cos[0], sin[0])):
        with pytest.raises(ValueError, match="rope"):
            make(a, b)
    with pytest.raises(ValueError, match="rope"):
        make(cos, sin, rotary_dim=32)                      # tables of another width
    make(cos, sin)
    make(None, None)


def test_row_orders_are_permutations(rt, case):
    import torch
    c, cache, cos, sin = case
    h = rt.Q4DecodeStep(cache, dev(c.table), dev(c.lens), 4, lens_host=c.lens, num_splits=2, row_order=[1, 0])
    q = dev(bits(np.random.default_rng(1), 2, 4, 64))
    want = h.attention(q)
    for bad in ([0], [0, 0], [0, 1, 2], [0, 2], [-1, 0], [[0, 1]], [0.5, 1.0], [], "longest"):
        with pytest.raises(ValueError, match="row_order"):
            h.plan(lens_host=c.lens, num_splits=2, row_order=bad)
        with pytest.raises(ValueError, match="row_order"):
            rt.Q4DecodeStep(cache, dev(c.table), dev(c.lens), 4, lens_host=c.lens, row_order=bad)
    assert torch.equal(h.attention(q), want)                # the plan from before still stands
    for good in ("auto", None, [0, 1], np.array([1, 0]), torch.tensor([1, 0])):
        h.plan(lens_host=c.lens, num_splits=2, row_order=good)
        assert torch.equal(h.attention(q), want)


def test_step_attends_over_the_token_that_it_appends(rt, case):
    # an object for attention over the cached tokens alone has no step: it would leave out the token just written
    c, cache, cos, sin = case
    rng = np.random.default_rng(2)
    q, k, v = (dev(bits(rng, 2, n, 64)) for n in (4, 2, 2))
    kw = dict(lens_host=c.lens, rope_cos=cos, rope_sin=sin)
    before = rt.Q4DecodeStep(cache, dev(c.table), dev(c.lens), 4, new_tokens=0, **kw)
    with pytest.raises(ValueError, match="new_tokens"):
        before.step(q, k, v)
    for n in (2, -1):
        with pytest.raises(ValueError, match="new_tokens"):
            rt.Q4DecodeStep(cache, dev(c.table), dev(c.lens), 4, new_tokens=n, **kw)
        with pytest.raises(ValueError, match="new_tokens"):
            kv = dev(bits(rng, 4, 16, 2, 64))
            rt.PagedAttention(kv, kv, dev(c.table.clip(0)), dev(c.lens), 4, lens_host=c.lens, new_tokens=n)
    before.attention(q)
    rt.Q4DecodeStep(cache, dev(c.table), dev(c.lens), 4, **kw).step(q, k, v)


def test_layouts(rt, case):
    c, cache, cos, sin = case
    with pytest.raises(ValueError, match="layout"):
        rt.Q4Cache(cache.k_codes, cache.v_codes, cache.params, layout="tokens")
    kv = dev(bits(np.random.default_rng(3), 4, 16, 2, 64))
    with pytest.raises(ValueError, match="layout"):
        rt.PagedAttention(kv, kv, dev(c.table), dev(c.lens), 4, layout="")
