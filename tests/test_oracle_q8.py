"""The 8-bit format's oracle against its definition written another way, and the bounds that the format promises."""
import numpy as np
import pytest

from oracle import q8_cache_oracle as Q
from oracle.paged_decode_oracle import bf16_to_f64, f64_to_bf16_rne


def test_e4m3_values_and_roundings_are_torch_s():
    torch = pytest.importorskip("torch")
    every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(Q.E4M3_VALUES, every, equal_nan=True)
    rng = np.random.default_rng(0)
    finite = Q.E4M3_VALUES[np.isfinite(Q.E4M3_VALUES)]
    ties = (np.sort(finite)[1:] + np.sort(finite)[:-1]) / 2
    y = np.concatenate([finite, ties, rng.standard_normal(20000) * np.exp2(rng.integers(-12, 8, 20000))]).clip(-448, 448).astype(np.float32)
    assert np.array_equal(Q.encode(y.astype(np.float64), Q.E4M3), torch.from_numpy(y).to(torch.float8_e4m3fn).view(torch.uint8).numpy())


@pytest.mark.parametrize("fmt", [Q.INT8, Q.E4M3])
def test_codes_are_the_nearest(fmt):
    rng = np.random.default_rng(1)
    values = np.unique(Q.code_values(np.arange(256, dtype=np.uint8), fmt))
    values = values[np.isfinite(values) & (np.abs(values) <= Q.LARGEST[fmt])]
    y = rng.uniform(-1.1, 1.1, 4000) * Q.LARGEST[fmt] * np.exp2(rng.integers(-8, 1, 4000))
    got = Q.code_values(Q.encode(y, fmt), fmt)
    near = np.abs(y[:, None].clip(-Q.LARGEST[fmt], Q.LARGEST[fmt]) - values[None]).min(1)
    assert np.array_equal(np.abs(got - y.clip(-Q.LARGEST[fmt], Q.LARGEST[fmt])), near)


@pytest.mark.parametrize("fmt", [Q.INT8, Q.E4M3])
def test_the_scale_is_the_least_that_suffices(fmt):
    m = np.array([[Q.LARGEST[fmt]]])
    for e in (-100, -7, 0, 60, Q.TOP[fmt]):
        assert Q.needed(m * 2.0**e, fmt) == 2.0**e
        if e < Q.TOP[fmt]:
            assert Q.needed(m * 2.0**e * (1 + 2.0**-7), fmt) == 2.0 ** (e + 1)
    assert Q.needed(np.zeros((1, 4)), fmt) == Q.needed(np.full((1, 1), 2.0**-130), fmt) == 2.0**-100
    assert np.isnan(Q.needed(np.array([[1.0, np.inf]]), fmt)) and np.isnan(Q.needed(np.array([[np.nan]]), fmt))
    top = bf16_to_f64(np.array([0x7F7F], dtype=np.uint16))
    assert np.isfinite(bf16_to_f64(f64_to_bf16_rne(Q.code_values(Q.encode(top / Q.needed(top[None], fmt), fmt), fmt) * Q.needed(top[None], fmt)))).all()


@pytest.mark.parametrize("fmt", [Q.INT8, Q.E4M3])
def test_values_appended_under_growing_scales_stay_within_a_step(fmt):
    """A growth at least doubles the scale, so the roundings of a code, half a step each, add up to less than one final step; for e4m3
    every rounding but the first is of a value that the format holds under twice the scale, unless it is below 2^-6 of it."""
    rng = np.random.default_rng(2)
    for _ in range(200):
        codes, s, given = np.zeros((16, 8), np.uint8), np.float32(np.nan), []
        for t in range(16):
            x = f64_to_bf16_rne(rng.standard_normal((1, 8)) * 2.0 ** rng.integers(-4, 5))
            s = Q.write(codes, s, x, t, fmt)
            given.append(bf16_to_f64(x)[0])
            err = np.abs(Q.code_values(codes[:t + 1], fmt) * s - np.array(given))
            assert (err < s * (1.0 if fmt == Q.INT8 else 2.0**-9 + 2.0**-4 * np.abs(given) / s)).all()


def test_a_block_written_at_once_and_in_two_parts_of_falling_size_is_the_same():
    rng = np.random.default_rng(3)
    for fmt in (Q.INT8, Q.E4M3):
        x = f64_to_bf16_rne(rng.standard_normal((16, 8)) * np.linspace(4, 1, 16)[:, None])
        x[0, 0] = 0x4180                                            # 16: the largest, in the first part
        one, two = np.zeros((16, 8), np.uint8), np.zeros((16, 8), np.uint8)
        s = Q.write(one, np.nan, x, 0, fmt)
        t = Q.write(two, np.nan, x[:5], 0, fmt)
        assert Q.write(two, t, x[5:], 5, fmt) == s == t and np.array_equal(one, two)
