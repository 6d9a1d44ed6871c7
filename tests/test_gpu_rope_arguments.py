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
