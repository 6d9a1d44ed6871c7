"""Arguments that the rotary object refuses."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rt():
    import torch
    from paper_2606_07665_b200 import build, runner
    build.build()
    torch.cuda.set_device(0)
    return runner


def test_rotary_rows_without_keys(rt):
    """An output for keys that are not given would come back unwritten."""
    import torch
    rope = rt.Rope.scaled(8, 64)
    q, k_out = torch.zeros(5, 4, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(5, 2, 64, dtype=torch.bfloat16, device="cuda")
    start, off = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.tensor([0, 5], dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError, match="k_out"):
        rope.rows(q, None, start, off, k_out=k_out)
    assert rope.rows(q, None, start, off)[1] is None


@pytest.mark.parametrize("which", ["q_norm_weight", "k_norm_weight"])
def test_rotary_norm_weights(rt, which):
    import torch
    cos, sin = (torch.zeros(8, 32, device="cuda") for _ in range(2))
    good = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    for bad in ([1.0] * 64, good.data_ptr(), 1.0):
        with pytest.raises(TypeError, match=which):
            rt.Rope(cos, sin, **{which: bad})
    for bad in (good.float(), good.cpu(), good[0], good.view(1, 64), torch.ones(128, dtype=torch.bfloat16, device="cuda")[::2]):
        with pytest.raises(ValueError, match=which):
            rt.Rope(cos, sin, **{which: bad})
    rt.Rope(cos, sin, **{which: good})
