"""4-bit attention at the ends of its stated range."""
import numpy as np
import pytest

from paper_2606_07665_b200 import workloads as W
from tests.test_gpu_q4 import Case, run_attention

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rt():
    import torch
    from paper_2606_07665_b200 import build, runner
    build.build()
    torch.cuda.set_device(0)
    return runner


@pytest.mark.parametrize("splits", [1, 3])
@pytest.mark.parametrize("Hq", [8, 24])
def test_values_as_large_as_the_sums_allow(rt, Hq, splits):
    """800 tokens of |V| below 2^108 are 2^118, the stated limit; scores that creep up by less than the reference's lag keep
    the weights as large as they get."""
    c = Case(rt, 130, [799], Hq, 2, 128, 16, 64, v_scale=2.0**105)
    q = W.f32_to_bf16_bits(np.abs(c.rng.standard_normal((1, Hq, 128))).astype(np.float32))
    for t in range(800):
        c.prm[c.table[0, t // 16], :, t % 16, 0, :, 1] = W.f32_to_bf16_bits(np.full((2, 2), -7.5 * 0.2 + 0.05 * t / 800, np.float32))
    top = max(np.abs(c.fetch(0, h, np.arange(800))[1]).max() for h in range(2))
    assert 2.0**106 < top and 800 * top < 2.0**118
    run_attention(rt, c, q=q, splits=splits)
