"""Rotation of many tokens per row and the scaled tables, against the oracle: rotations bit for bit."""
import numpy as np
import pytest

from oracle import paged_decode_oracle as O
from oracle import q8_cache_oracle as Q
from paper_2606_07665_b200 import workloads as W

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rt():
    import torch
    from paper_2606_07665_b200 import build, runner
    build.build()
    torch.cuda.set_device(0)
    return runner


def bits(rng, *shape, scale=1.0):
    return W.f32_to_bf16_bits((rng.standard_normal(shape) * scale).astype(np.float32))


def dev(a):
    import torch
    a = np.ascontiguousarray(a)
    return torch.from_numpy(a.view(np.int16) if a.dtype == np.uint16 else a).cuda()


def host(t):
    return t.cpu().numpy().view(np.uint16)


def reference(x, start, off, cos, sin, R, interleaved, w, untouched):
    out = untouched.copy()
    for b in range(len(start)):
        for i in range(off[b], off[b + 1] if start[b] >= 0 else off[b]):
            p = int(start[b]) + i - int(off[b])
            if p >= len(cos):
                continue
            for h in range(x.shape[1]):
                y = x[i, h] if w is None else O.rms_norm_bf16(x[i, h], w, 1e-5)
                out[i, h] = O.rope_rotate_variant_bf16(y, cos[p], sin[p], R, interleaved)
    return out


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("R", [None, 2, 16, 18, 32, 40, 50, 64])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (5, 0), (7, 3)])
def test_rows(rt, d, R, interleaved, norm, Hq, Hkv):
    import torch
    R = R or d
    rng = np.random.default_rng(R + d)
    lens, start = [3, 0, 1, 5, 0, 2], np.array([0, 4, 77, -1, 2, 9], dtype=np.int32)
    off = 1 + np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    total = int(off[-1]) + 2                                        # tokens in front and behind belong to no row
    cos, sin = W.rope_table(80, R, 10000.0)
    w = (bits(rng, d), bits(rng, d)) if norm else (None, None)
    rope = rt.Rope(dev(cos), dev(sin), interleaved=interleaved, norm_eps=1e-5, q_norm_weight=None if w[0] is None else dev(w[0]),
                   k_norm_weight=None if w[1] is None else dev(w[1]))
    joint = bits(rng, total, Hq + 2 * Hkv + 1, d)
    dj = dev(joint)
    q, k = dj[:, :Hq], dj[:, Hq:Hq + Hkv] if Hkv else None
    q_out, k_out = dev(bits(rng, total, Hq, d)), dev(bits(rng, total, Hkv, d)) if Hkv else None
    had = host(q_out).copy(), host(k_out).copy() if Hkv else None
    got = rope.rows(q, k, dev(start), dev(off), q_out=q_out, k_out=k_out)
    torch.cuda.synchronize()
    assert int(rope.status_flag) == 0
    assert np.array_equal(host(got[0]), reference(joint[:, :Hq], start, off, cos, sin, R, interleaved, w[0], had[0]))
    if Hkv:
        assert np.array_equal(host(got[1]), reference(joint[:, Hq:Hq + Hkv], start, off, cos, sin, R, interleaved, w[1], had[1]))
    assert np.array_equal(host(dj), joint)
    rope.rows(q, k, dev(start), dev(off), q_out=q, k_out=k)         # in place, in the joint tensor
    torch.cuda.synchronize()
    want = joint.copy()
    want[:, :Hq] = reference(joint[:, :Hq], start, off, cos, sin, R, interleaved, w[0], joint[:, :Hq])
    if Hkv:
        want[:, Hq:Hq + Hkv] = reference(joint[:, Hq:Hq + Hkv], start, off, cos, sin, R, interleaved, w[1], joint[:, Hq:Hq + Hkv])
    assert np.array_equal(host(dj), want)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("kind", ["ranges", "cancel", "zeros", "extremes"])
def test_values_that_need_more_than_fp32(rt, interleaved, kind):
    """Magnitudes far apart, sums that cancel to a few bits, zeros of both signs, subnormals and the largest values."""
    import torch
    rng = np.random.default_rng(3)
    T, H, d = 400, 4, 128
    cos, sin = W.rope_table(T, d, 10000.0)
    x = rng.standard_normal((T, H, d))
    if kind == "ranges":
        x = np.ldexp(x, rng.integers(-130, 120, (T, H, d)))
    elif kind == "cancel":                                          # x_first ~ x_second tan(angle): the first result is nearly 0
        half = np.arange(d // 2)
        first, second = (2 * half, 2 * half + 1) if interleaved else (half, half + d // 2)
        x[..., first] = x[..., second] * (sin / cos).astype(np.float64)[:, None]
    elif kind == "zeros":
        x = np.where(rng.random((T, H, d)) < 0.5, np.copysign(0.0, x), x)
    xb = W.f32_to_bf16_bits(x.astype(np.float32))
    if kind == "extremes":
        xb = rng.choice(np.array([0x0001, 0x8001, 0x007F, 0x0080, 0x7F7F, 0xFF7F, 0x7F00, 0x3F80, 0x0000, 0x8000], dtype=np.uint16), (T, H, d))
    rope = rt.Rope(dev(cos), dev(sin), interleaved=interleaved)
    out, _ = rope.rows(dev(xb), None, dev(np.zeros(1, np.int32)), dev(np.array([0, T], np.int32)))
    torch.cuda.synchronize()
    want = reference(xb, [0], [0, T], cos, sin, d, interleaved, None, xb)
    at = np.argwhere(host(out) != want)
    assert not len(at), (len(at), at[:3].tolist(), hex(host(out)[tuple(at[0])]), hex(want[tuple(at[0])]))


@pytest.mark.parametrize("B", [1, 31, 32, 33, 1000, 1025, 3000])
def test_many_rows(rt, B):
    """The search for a token's row, with runs of empty rows, at every size of a round of it."""
    import torch
    rng = np.random.default_rng(B)
    lens = rng.integers(0, 4, B) * (rng.random(B) < 0.5)
    off = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    start = rng.integers(-1, 50, B).astype(np.int32)
    T = int(off[-1]) + 1
    cos, sin = W.rope_table(60, 64, 10000.0)
    x = bits(rng, T, 1, 64)
    rope = rt.Rope(dev(cos), dev(sin))
    out = dev(x).clone()
    rope.rows(dev(x), None, dev(start), dev(off), q_out=out)
    torch.cuda.synchronize()
    assert np.array_equal(host(out), reference(x, start, off, cos, sin, 64, False, None, x))


def test_positions_past_the_table(rt):
    import torch
    from paper_2606_07665_b200 import binding as ac
    rng = np.random.default_rng(1)
    cos, sin = W.rope_table(10, 64, 10000.0)
    rope = rt.Rope(dev(cos), dev(sin))
    x = bits(rng, 12, 3, 64)
    start, off = np.array([7, 2**31 - 3], dtype=np.int32), np.array([0, 6, 12], dtype=np.int32)
    out = dev(x).clone()
    rope.rows(dev(x), None, dev(start), dev(off), q_out=out)
    torch.cuda.synchronize()
    assert int(rope.status_flag) == ac.AC_FLAG_POSITION_OOB
    assert np.array_equal(host(out), reference(x, start, off, cos, sin, 64, False, None, x))


def test_one_token_of_many_heads_and_many_tokens(rt):
    """Both ends of how the heads of a token are shared out among warps."""
    import torch
    rng = np.random.default_rng(2)
    for T, Hq, Hkv, d in ((1, 200, 8, 128), (1, 1, 1, 64), (6000, 3, 1, 64), (5000, 9, 2, 128)):
        cos, sin = W.rope_table(T + 5, d, 500000.0)
        q, k = bits(rng, T, Hq, d), bits(rng, T, Hkv, d)
        rope = rt.Rope(dev(cos), dev(sin))
        qo, ko = rope.rows(dev(q), dev(k), dev(np.array([5], np.int32)), dev(np.array([0, T], np.int32)))
        torch.cuda.synchronize()
        some = np.unique(rng.integers(0, T, 40))
        for t in some:
            for x, y in ((q, qo), (k, ko)):
                got = host(y)[t]
                for h in range(x.shape[1]):
                    assert np.array_equal(got[h], O.rope_rotate_variant_bf16(x[t, h], cos[t + 5], sin[t + 5], d, False)), (t, h)


SCALINGS = [dict(), dict(scaling="linear", factor=4.0), dict(scaling="base", factor=8.0),
            dict(scaling="ramp", factor=32.0, original=8192, low=1.0, high=4.0, magnitude=0.1 * np.log(32.0) + 1),
            dict(scaling="ramp", factor=8.0, original=4096, low=1.0, high=32.0)]


@pytest.mark.parametrize("how", SCALINGS)
@pytest.mark.parametrize("R,positions,first", [(4, 1, 0), (18, 63, 0), (64, 65, 1000000), (128, 1000, 130000), (128, 70000, 0), (6, 7, 2**31)])
def test_tables(rt, how, R, positions, first):
    """The angle is p f with f from a power (2^-51), one product (2^-53) and the blend (2^-51): below 2^-49 of it.  The
    rotation from the run's first position adds 64 * 2^-52, the multiplication by the magnitude 2^-53; then one rounding to
    fp32, 2^-24 of the value."""
    import torch
    base = 500000.0
    rope = rt.Rope.scaled(positions, R, base=base, **how)
    if first:
        rope.fill(first, base=base, **how)
    torch.cuda.synchronize()
    m = how.get("magnitude", 1.0)
    f = Q.frequencies(R, base, **{k: v for k, v in how.items() if k != "magnitude"})
    c, s = Q.tables(first, positions, f, m)
    angle = ((first + np.arange(positions, dtype=np.float64))[:, None] * f.astype(np.float64)[None, :])
    for got, want in ((rope.cos, c), (rope.sin, s)):
        err = np.abs(got.cpu().numpy().astype(np.longdouble) - want)
        bound = 2.0**-24 * np.abs(want) * (1 + 2.0**-20) + m * (angle * 2.0**-49 + 2.0**-45) + 2.0**-150
        assert (err <= bound).all(), float((err / bound).max())


def test_fill_writes_nothing_else(rt):
    import torch
    t = torch.full((2, 12, 9), 7.0, device="cuda")
    held = t.clone()
    rope = rt.Rope(t[0, 4:8].contiguous(), t[1, 4:8].contiguous())
    big = torch.full((2, 4 * 9 + 64), 7.0, device="cuda")
    rope = rt.Rope(big[0, :36].view(4, 9), big[1, 32 - 32:36].view(4, 9))
    rope.fill(3)
    torch.cuda.synchronize()
    assert (big[:, 36:] == 7).all() and (big[:, :36] != 7).all() and torch.equal(t, held)


def test_rotation_feeds_the_decode_step(rt):
    """A prompt rotated here and the same tokens appended one by one hold the same keys (bf16 queries out are equal)."""
    import torch
    rng = np.random.default_rng(6)
    n, Hq, Hkv, d, ps = 40, 8, 2, 128, 16
    rope = rt.Rope.scaled(64, d, base=10000.0, scaling="ramp", factor=4.0, original=32, low=1.0, high=4.0, magnitude=1.1, interleaved=True)
    q, k = dev(bits(rng, n, Hq, d)), dev(bits(rng, n, Hkv, d))
    q_rot, k_rot = rope.rows(q, k, dev(np.zeros(1, np.int32)), dev(np.array([0, n], np.int32)))
    table, lens = dev(np.array([[2, 0, 1]], np.int32)), torch.zeros(1, dtype=torch.int32, device="cuda")
    caches = [rt.Q4Cache.empty(3, ps, Hkv, d) for _ in range(2)]
    step = rt.Q4DecodeStep(caches[0], table, lens, Hq, max_context_len=64, rope_cos=rope.cos, rope_sin=rope.sin,
                           rope_variants=dict(interleaved=True))
    for t in range(n):
        assert torch.equal(step.append(q[t:t + 1], k[t:t + 1], k[t:t + 1])[0], q_rot[t])
        lens += 1
    lens.zero_()
    caches[1].store(k_rot, k, table, lens, dev(np.array([0, n], np.int32)))
    assert torch.equal(caches[0].k_codes, caches[1].k_codes) and torch.equal(caches[0].params, caches[1].params)


@pytest.mark.parametrize("d,Hq,Hkv,T,R,interleaved,norm", [(128, 17, 1, 12000, 128, False, False), (128, 17, 3, 12000, 64, True, False),
                                                           (64, 33, 5, 13000, 32, False, True), (64, 40, 0, 12000, 64, True, True)])
def test_a_call_of_many_tokens_is_its_pieces(rt, d, Hq, Hkv, T, R, interleaved, norm):
    """Calls of 48 MB and more take another kernel: the same bits, also in place, with rows that are inactive, empty, past the table."""
    import torch
    from paper_2606_07665_b200 import binding as ac
    assert T * (Hq + Hkv) * d * 2 >= 48 << 20
    rng = np.random.default_rng(7)
    cut = np.sort(rng.integers(5, T - 5, 40))
    off = np.concatenate([[5], cut, cut[-1:], [T - 5]]).astype(np.int32)        # one row is empty; tokens of no row at both ends
    start = rng.integers(0, 50, len(off) - 1).astype(np.int32)
    start[7], start[20] = -1, 19_000
    rope = rt.Rope.scaled(20_000, R, interleaved=interleaved, norm_eps=1e-5, q_norm_weight=dev(bits(rng, d)) if norm else None)
    q, k = torch.randn(T, Hq, d, device="cuda").bfloat16(), torch.randn(T, Hkv, d, device="cuda").bfloat16()
    q[100:200] = 0
    q[300, 0, :4] = torch.tensor([float("inf"), float("nan"), 1e38, -0.0])
    q_out, k_out = torch.full_like(q, 7.0), torch.full_like(k, 7.0)
    want_q, want_k = q_out.clone(), k_out.clone()
    k_, ko_ = (k, k_out) if Hkv else (None, None)
    rope.rows(q, k_, dev(start), dev(off), q_out=q_out, k_out=ko_)
    same = lambda a, b: torch.equal(a.view(torch.int16), b.view(torch.int16))      # noqa: E731
    for b in range(len(start)):                                     # each row by itself, from a view that begins with it
        lo, hi = int(off[b]), int(off[b + 1])
        if hi > lo:
            rope.rows(q[lo:hi], k[lo:hi] if Hkv else None, dev(start[b:b + 1]), dev(np.array([0, hi - lo], np.int32)), q_out=want_q[lo:hi],
                      k_out=want_k[lo:hi] if Hkv else None)
    assert same(q_out, want_q) and same(k_out, want_k)
    assert int(rope.status_flag) in (0, ac.AC_FLAG_POSITION_OOB)
    rope.rows(q, k_, dev(start), dev(off), q_out=q, k_out=k_)
    untouched = torch.ones(T, dtype=torch.bool, device="cuda")
    for b in range(len(start)):
        if start[b] >= 0:
            untouched[int(off[b]):int(off[b]) + max(0, min(int(off[b + 1] - off[b]), 20_000 - int(start[b])))] = False
    assert same(q[~untouched], want_q[~untouched]) and same(k[~untouched], want_k[~untouched])
    assert (want_q[untouched] == 7).all() and not (want_q[~untouched][:, 0] == 7).all(-1).any()
    torch.cuda.synchronize()
