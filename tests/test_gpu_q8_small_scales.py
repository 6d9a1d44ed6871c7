"""8-bit attention where V's scales are far below those that the library writes: the stated accuracy holds there too."""
import numpy as np
import pytest

from oracle import q8_cache_oracle as Q
from tests.test_gpu_q8 import dev, f64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rt():
    import torch
    from paper_2606_07665_b200 import build, runner
    build.build()
    torch.cuda.set_device(0)
    return runner


@pytest.mark.parametrize("fmt", [Q.INT8, Q.E4M3])
@pytest.mark.parametrize("exponent", [-100, -113, -114, -117, -120])
@pytest.mark.parametrize("weight", [8.0, 15.3, 21.5])
@pytest.mark.parametrize("splits", [1, 3])
def test_light_tokens_beside_a_heavy_one(rt, fmt, exponent, weight, splits):
    """One token of weight 1 whose value is zero, 8000 of weight 2^-`weight` under one scale s = 2^exponent.  Each light weight times s
    is off by 2^-11 of itself or by 2^-31 s, and the result, a normal bf16, by its rounding, 2^-8."""
    import torch
    n, d, block = 8001, 64, 16
    cache = rt.Q8Cache.empty(-(-n // 64), 64, 1, d, block, torch.int8 if fmt == Q.INT8 else torch.float8_e4m3fn)
    cache.scales[..., 0] = 1.0
    cache.scales[..., 1] = 2.0**exponent
    cache.v_codes.fill_(100.0 if fmt == Q.INT8 else 96.0)
    cache.v_codes.view(torch.uint8)[0, 0] = 0
    cache.k_codes[0, 0, 0, 0] = 1.0                                 # score 1 times the softmax scale, the others 0
    q = np.zeros((1, 4, d), dtype=np.uint16)
    q[..., 0] = 0x3F80
    table = torch.arange(cache.num_pages, dtype=torch.int32, device="cuda").view(1, -1)
    lens = torch.full((1,), n, dtype=torch.int32, device="cuda")
    step = rt.Q8DecodeStep(cache, table, lens, 4, lens_host=[n], num_splits=splits, softmax_scale=weight * np.log(2.0), new_tokens=0)
    got = f64(step.attention(dev(q)))
    light = 2.0**-weight
    value = (100.0 if fmt == Q.INT8 else 96.0) * 2.0**exponent
    total = 1 + (n - 1) * light
    want = (n - 1) * light * value / total
    assert want > 2.0**-126
    # the softmax scale as fp32 times log2 e: 2^-22 of a score of up to 21.5 powers of two; fp32 sums: 2^-14
    off = max(2.0**-11, 2.0**-31 / light) + 2.0**-13
    assert (np.abs(got - want) <= want * (off + 2.0**-8 * (1 + 2.0**-8))).all(), float(np.abs(got / want - 1).max() / (off + 2.0**-8))
