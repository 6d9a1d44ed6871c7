"""Scalings whose tables would hold no numbers: refused on the host, before any device is touched."""
import pytest

SHAPE = 2
P = 1 << 20                                       # a pointer that is never followed
INF = float("inf")


@pytest.fixture(scope="module")
def ac():
    from paper_2606_07665_b200 import binding, build
    build.build()
    return binding


def status(ac, how, first=0, positions=0, rotary=64):
    return ac.lib().ac_rope_tables(P, P, first, positions, rotary, how, None)


def test_numbers_beyond_the_largest(ac):
    s = ac.rope_scaling
    ramp = dict(kind=ac.AC_ROPE_RAMP, factor=2.0, original=10.0)
    for bad in (s(magnitude=INF), s(base=INF), s(kind=ac.AC_ROPE_LINEAR, factor=INF), s(low=-INF, high=2.0, **ramp), s(low=1.0, high=INF, **ramp),
                s(low=-1.5e308, high=1.5e308, **ramp), s(low=1.0, high=2.0, **dict(ramp, original=INF))):
        assert status(ac, bad) == SHAPE
    for good in (s(magnitude=1e300), s(low=-1e300, high=1e300, **ramp), s(low=1.0, high=4.0, **ramp), s(low=INF), s(factor=INF)):
        assert status(ac, good) != SHAPE          # (the last two are not used)


def test_a_larger_base_that_is_no_number(ac):
    how = lambda factor, base=1e4: ac.rope_scaling(base=base, kind=ac.AC_ROPE_BASE, factor=factor)      # noqa: E731
    assert status(ac, how(1e200), rotary=4) == SHAPE and status(ac, how(1e-200), rotary=4) == SHAPE      # squared
    assert status(ac, how(1e250, 1e100)) == SHAPE
    assert status(ac, how(1e200), rotary=128) != SHAPE and status(ac, how(8.0), rotary=4) != SHAPE


def test_positions_beyond_the_last(ac):
    how = ac.rope_scaling()
    assert status(ac, how, 2**63 - 5, 5) == SHAPE
    assert status(ac, how, 2**63 - 1, 1) == SHAPE and status(ac, how, 2**63 - 6, 5) != SHAPE
