"""Tables of as many positions as the call takes."""
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


@pytest.mark.parametrize("positions", [2**31 - 1, 2**31 - 31])
def test_the_most_positions(rt, positions):
    """One frequency, 1: cosines and sines of the positions themselves.  A position below 2^31 is exact, its cosine within 2^-45
    of a table's (a run of 32 rotations), and rounded to fp32."""
    import torch
    cos, sin = (torch.full((positions, 1), 7.0, device="cuda") for _ in range(2))
    rt.Rope(cos, sin).fill()
    torch.cuda.synchronize()
    rng = np.random.default_rng(1)
    at = np.unique(np.concatenate([np.arange(70), rng.integers(0, positions, 5000), positions - 1 - np.arange(70)]))
    picked = torch.from_numpy(at).cuda()
    for table, f in ((cos, np.cos), (sin, np.sin)):
        want = f(at.astype(np.longdouble))
        err = np.abs(table[picked, 0].cpu().numpy().astype(np.longdouble) - want)
        assert (err <= 2.0**-24 * np.abs(want) * (1 + 2.0**-20) + 2.0**-44).all()
        for piece in table.view(-1).split(1 << 28):
            assert bool((piece.abs() <= 1).all())                   # every one is written
    del cos, sin, table, piece
    torch.cuda.empty_cache()
