"""Rotary rows normalise to the bits of the decode step's append, also where the sum of squares depends on its order."""
import numpy as np
import pytest

from paper_2606_07665_b200 import workloads as W

pytestmark = pytest.mark.gpu

VECTORS = 3000


@pytest.fixture(scope="module")
def rt():
    import torch
    from paper_2606_07665_b200 import build, runner
    build.build()
    torch.cuda.set_device(0)
    return runner


def bf16_below(x):
    """The largest bf16 value that is not above x > 0."""
    m, e = np.frexp(x)
    return float(np.ldexp(np.floor(m * 256.0), e - 8))


def on_the_border(rng, d):
    """A vector with an element 2^-k that its norm brings to within an ulp or two of fp64 of the middle of two bf16 values, and
    whose smaller elements have squares below half an ulp of the sum: which of them count depends on the order of the additions."""
    middle = 1 + (2 * rng.integers(0, 128) + 1) / 256.0
    total = d / (middle * middle)
    ulp = np.spacing(total)
    x, at, i = np.zeros(d), (rng.permutation(d) if rng.random() < 0.5 else np.arange(d)), 1
    x[at[0]] = 2.0 ** -rng.integers(1, 6)
    rest = total - x[at[0]] ** 2 - rng.uniform(0, 60) * ulp
    while rest > 4 * ulp and i < 12:
        x[at[i]] = bf16_below(np.sqrt(rest))
        rest -= x[at[i]] ** 2
        i += 1
    small = np.sqrt(rng.uniform(0.05, 0.6) * ulp)
    for j in range(i, d):
        x[at[j]] = bf16_below(small * rng.uniform(0.8, 1.2))
    return x * np.where(rng.random(d) < 0.5, -1, 1)


def crosswise(x):
    """The sum of squares as the append kernels form it: d/32 neighbours at a time, these sums joined at distances 16, 8, 4, 2, 1."""
    n = len(x) // 32
    p = np.zeros(32)
    for e in range(n):
        p = p + x.reshape(32, n)[:, e] ** 2
    for off in (16, 8, 4, 2, 1):
        p = p + p[np.arange(32) ^ off]
    return p[0]


def normalised(x, total):
    y = x * (1.0 / np.sqrt(total / len(x)))
    m, e = np.frexp(y)
    return np.ldexp(np.rint(m * 256.0), e - 8)                      # nearest-even bf16


@pytest.fixture(scope="module", params=[64, 128])
def borders(request):
    """Vectors, what becomes of them, and how many of them another order would change."""
    rng = np.random.default_rng(request.param)
    xs = [on_the_border(rng, request.param) for _ in range(VECTORS)]
    want = [normalised(x, crosswise(x)) for x in xs]
    other = sum(not np.array_equal(w, normalised(x, np.cumsum(x * x)[-1])) for x, w in zip(xs, want))
    assert other > 20
    bits = lambda a: W.f32_to_bf16_bits(np.array(a, dtype=np.float32))      # noqa: E731
    return request.param, bits(xs), bits(want)


def dev(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a).view(np.int16)).cuda().view(torch.bfloat16)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("part", [1, 2, 4])
@pytest.mark.parametrize("many", [False, True])
def test_rows(rt, borders, interleaved, part, many):
    """At position 0 the rotation is none, so that the results are the normalised vectors.  Few tokens, and as many as take the
    streaming kernel."""
    import torch
    d, x, want = borders
    times = -(-(32 << 20) // (VECTORS * d * 2)) if many else 1
    q = dev(x).view(VECTORS // 10, 10, d).repeat(times, 1, 1)
    T = q.shape[0]
    one = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    rope = rt.Rope.scaled(4, d // part, interleaved=interleaved, q_norm_weight=one, k_norm_weight=one)
    start, off = torch.zeros(T, dtype=torch.int32, device="cuda"), torch.arange(T + 1, dtype=torch.int32, device="cuda")
    got = rope.rows(q, q, start, off)
    ref = dev(want).view(VECTORS // 10, 10, d).repeat(times, 1, 1)
    assert int(rope.status_flag) == 0
    for g in got:
        differ = (g != ref).any(-1)
        assert not bool(differ.any()), int(differ.sum())


def test_append(rt, borders):
    """What the rows are compared with is what the append gives."""
    import torch
    d, x, want = borders
    n = VECTORS // 10
    one = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    rope = rt.Rope.scaled(4, d)
    table, lens = torch.arange(n, dtype=torch.int32, device="cuda").view(n, 1), torch.zeros(n, dtype=torch.int32, device="cuda")
    for cache, kind in ((rt.Q4Cache.empty(n, 16, 1, d), rt.Q4DecodeStep), (rt.Q8Cache.empty(n, 16, 1, d), rt.Q8DecodeStep)):
        step = kind(cache, table, lens, 10, max_context_len=16, rope_cos=rope.cos, rope_sin=rope.sin,
                    rope_variants=dict(q_norm_weight=one, k_norm_weight=one, norm_eps=0.0))
        got = step.append(dev(x).view(n, 10, d), *(torch.ones(n, 1, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)))
        assert torch.equal(got.view(-1, d), dev(want))
