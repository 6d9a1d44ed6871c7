"""Tables of as many positions as the call takes, and of positions far out."""
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


@pytest.mark.parametrize("base,R", [(500000.0, 128), (1e6, 106), (1e6, 18), (10000.0, 94), (30.0, 64), (1e8, 6)])
@pytest.mark.parametrize("how", [dict(), dict(scaling="linear", factor=3.0), dict(scaling="base", factor=40.0), dict(scaling="ramp", factor=40.0, original=8192.0, low=1.0, high=4.0),
                                 dict(scaling="ramp", factor=0.3, original=50.0, low=0.0, high=1.0)])
@pytest.mark.parametrize("first", [2**30, 2**36])
def test_the_angle_of_far_positions(rt, base, R, how, first):
    """So far out that the angle's error is most of the entry's.  f = base^e: e = -2i/R is rounded, 2^-53 |e ln base| of f, and the power
    is off by 2 ulp, 4 * 2^-53; the larger base's logarithm by (2 |ln factor| + 3) 2^-53; a division or the turns, and the product with
    the position, add up to five roundings.  A blend of g = (turns - low) / (high - low) moves by the turns' error times
    high / (high - low), and f by at most that times max(factor, 1/factor).  The reference's angle is off by less than 2^-60 of it."""
    from oracle import q8_cache_oracle as Q
    n = 40
    rope = rt.Rope.scaled(n, R, base=base)
    rope.fill(first, base=base, **how)
    f = Q.frequencies(R, base, **how)
    c, s = Q.tables(first, n, f)
    factor = how.get("factor", 1.0)
    large = base * factor ** (R / (R - 2)) if how.get("scaling") == "base" else base
    off = (abs(np.log(large)) + 2 * abs(np.log(factor)) + 12) * 2.0**-53
    if how.get("scaling") == "ramp":
        off *= max(factor, 1 / factor) * how["high"] / (how["high"] - how["low"])
    angle = (first + np.arange(n, dtype=np.float64))[:, None] * f.astype(np.float64)[None, :]
    for got, want in ((rope.cos, c), (rope.sin, s)):
        err = np.abs(got.cpu().numpy().astype(np.longdouble) - want)
        bound = 2.0**-24 * np.abs(want) * (1 + 2.0**-20) + angle * (off * (1 + 2.0**-40) + 2.0**-60) + 2.0**-45 * (1 + 2.0**-20)
        assert (err <= bound).all(), float((err / bound).max())
