"""The 8-bit cache on the GPU against its oracle: codes and scales are compared one by one, attention within a bound derived
from its roundings."""
import numpy as np
import pytest

from oracle import paged_decode_oracle as O
from oracle import q4_cache_oracle as A
from oracle import q8_cache_oracle as Q
from paper_2606_07665_b200 import workloads as W

pytestmark = pytest.mark.gpu

FORMATS = [Q.INT8, Q.E4M3]


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
    import torch
    if t.dtype == torch.bfloat16:
        t = t.view(torch.int16)
    if t.dtype in (torch.int8, torch.float8_e4m3fn):
        t = t.view(torch.uint8)
    a = t.cpu().numpy()
    return a.view(np.uint16) if a.dtype == np.int16 else a


def f64(t):
    return O.bf16_to_f64(host(t))


class Case:
    """A cache of normal values under a scattered block table; the scales of everything that no row holds are NaN, and its
    codes, as those behind a row's end, the pattern 0x7F (NaN, for e4m3)."""

    def __init__(self, seed, lens, Hq, Hkv, d, ps, block, fmt, layout="token_major", room=1, spare=3, exponents=(-6, -3)):
        rng = self.rng = np.random.default_rng(seed)
        self.lens = np.asarray(lens, dtype=np.int32)
        self.B, self.Hq, self.Hkv, self.d, self.ps, self.block, self.fmt, self.layout = len(lens), Hq, Hkv, d, ps, block, fmt, layout
        need = [-(-(max(int(n), 0) + room) // ps) for n in lens]
        self.num_pages = sum(need) + spare
        perm = rng.permutation(self.num_pages)
        self.table = np.full((self.B, max(need) + 1), -7, dtype=np.int32)      # unused entries name no page at all
        at = 0
        k, v = (np.full((self.num_pages, ps, Hkv, d), 0x7F, dtype=np.uint8) for _ in range(2))
        scales = np.full((self.num_pages, Hkv, ps // block, 2), np.nan, dtype=np.float32)
        for b, n in enumerate(need):
            self.table[b, :n] = perm[at:at + n]
            at += n
            tokens = int(lens[b]) + room if lens[b] >= 0 else 0
            t = np.arange(tokens)
            for pool in (k, v):
                y = rng.standard_normal((tokens, Hkv, d)) * (32.0 if fmt == Q.INT8 else 64.0)
                pool[self.table[b, t // ps], t % ps] = Q.encode(y, fmt)
            for blk in range(-(-tokens // block)):
                e = rng.integers(*exponents, (Hkv, 2))
                scales[self.table[b, blk * block // ps], :, blk * block % ps // block] = np.ldexp(np.float32(1), e)
        self.cache = Q.Cache(k, v, scales, fmt)

    def upload(self, rt):
        import torch
        move = (lambda x: x) if self.layout == "token_major" else (lambda x: x.transpose(0, 2, 1, 3))
        kind = torch.int8 if self.fmt == Q.INT8 else torch.float8_e4m3fn
        c = rt.Q8Cache.empty(self.num_pages, self.ps, self.Hkv, self.d, self.block, kind, self.layout)
        c.k_codes.view(torch.uint8).copy_(dev(move(self.cache.pools[0])))
        c.v_codes.view(torch.uint8).copy_(dev(move(self.cache.pools[1])))
        c.scales.copy_(dev(self.cache.scales))
        return c

    def same(self, c, but=None):
        """The device's cache is the oracle's, except for the codes of blocks whose scale is NaN."""
        move = (lambda x: x) if self.layout == "token_major" else (lambda x: x.transpose(0, 2, 1, 3))
        s = host(c.scales)
        at = np.argwhere(~((s == self.cache.scales) | (np.isnan(s) & np.isnan(self.cache.scales))))
        assert not len(at), ("scales", at[:4].tolist(), s[tuple(at[0])], self.cache.scales[tuple(at[0])])
        for side, pool in enumerate((c.k_codes, c.v_codes)):
            got, want = move(host(pool)), self.cache.pools[side]
            fine = ~np.isnan(s[..., side]).transpose(0, 2, 1).repeat(self.block, 1)          # [page, slot, head]
            at = np.argwhere((got != want) & fine[..., None])
            assert not len(at), ("codes", side, len(at), at[:4].tolist(), got[tuple(at[0])], want[tuple(at[0])])

    def fetch(self, b, h, t):
        K, V = (self.cache.read(side, self.table[b], t, h) for side in (0, 1))
        return K, V, np.abs(V)

    def floor(self, n, window=0, sinks=0):
        """A weight times V's scale below 2^-14 is rounded to a multiple of 2^-24 in fp16: an error of 2^-25, in units in which the
        largest scale of V that the row attends over is at least 2^6, before a division by at least 1 (the reference of the
        weights is at most their maximum): 2^-31 of that scale times the code, per token.  [B, Hq, d]"""
        out = np.zeros((self.B, self.Hkv, self.d))
        for b in range(self.B):
            t = A.visible(int(n[b]), window, sinks)
            if t.size:
                page, slot = self.table[b, t // self.ps], t % self.ps
                c = np.abs(Q.code_values(self.cache.pools[1][page, slot], self.fmt))
                top = self.cache.scales[page, :, slot // self.block, 1].max(0).astype(np.float64)
                out[b] = 2.0**-31 * top[:, None] * c.sum(0)
        return out.repeat(self.Hq // self.Hkv, 1)


def check(got, ref, room, what, floor=0.0):
    """Each weight times V's scale is rounded to fp16, 2^-11 relative, so the result moves by at most 2^-11 sum_t p_t |V_t|
    (`room`).  Scores are sums of d <= 128 products in eight steps of the tensor pipe, each losing at most 2^-22 of the
    magnitudes added up (at most 48 powers of two in these tests): 2^-14 of each weight, twice with the normaliser.  The fp32 sums over
    tokens lose less than 2^-14 at these lengths.  `floor`: Case.floor.  The result is rounded to bf16, 2^-8 relative."""
    bound = 2.0**-8 * np.abs(ref) * (1 + 2.0**-8) + (2.0**-11 + 2.0**-12) * room + floor + 1e-30
    err = np.abs(got - ref)
    assert np.isfinite(got).all(), what
    assert (err <= bound).all(), (what, float((err / bound).max()))
    return float((err / bound).max())


def run_attention(rt, c, window=0, sinks=0, splits=None, q=None, new_tokens=1, q_scale=1.0, slack=1, **kw):
    import torch
    q = bits(c.rng, c.B, c.Hq, c.d, scale=q_scale) if q is None else q
    cache = c.upload(rt)
    h = rt.Q8DecodeStep(cache, dev(c.table), dev(c.lens), c.Hq, lens_host=c.lens, window=window, sinks=sinks, num_splits=splits,
                        new_tokens=new_tokens, **kw)
    out = h.attention(dev(q))
    again = h.attention(dev(q))
    torch.cuda.synchronize()
    assert torch.equal(out, again), "two calls differ"
    assert int(h.status_flag) == 0
    n = np.where(c.lens >= 0, c.lens + new_tokens, 0)
    ref, room = A.attention(q, c.fetch, n, c.Hkv, window, sinks, slack=True)
    check(f64(out), ref, room * slack, f"splits {h.num_splits}", c.floor(n, window, sinks))
    assert not f64(out)[n <= 0].any()
    return h, out


# ---- writing ---------------------------------------------------------------------------------------------------


def with_specials(rng, x):
    """Puts into the first tokens: an infinity, NaN, both zeros, subnormals, the type's extremes, values at a tie."""
    x = x.copy()
    flat = x.reshape(-1, x.shape[-1])
    for i, vals in ((0, [0x0000, 0x8000]), (1, [0x0001, 0x8003, 0x0007]), (5, [0x7F7F, 0xFF7F, 0x7E80, 0x0000]),
                    (9, [0x4170, 0x3F00, 0x3FC0, 0x4020, 0xBF00]), (len(flat) - 1, [0x3F80, 0x7F80]), (len(flat) // 2, [0x7FC0, 0x3F80])):
        if 0 <= i < len(flat):
            flat[i] = np.resize(np.array(vals, dtype=np.uint16), x.shape[-1])
    return x


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d,ps,block", [(128, 16, 16), (64, 48, 16), (128, 64, 32), (64, 64, 64), (128, 96, 48), (64, 256, 256)])
@pytest.mark.parametrize("layout", ["token_major", "head_major"])
@pytest.mark.parametrize("heads,lens,specials", [(1, [0], False), (3, [5, 0, 0, 33, 64], False), (8, [100, 1, 17], True),
                                                 (2, [3, 0, 18, 300], True)])
def test_store_and_load(rt, fmt, d, ps, block, layout, heads, lens, specials):
    import torch
    rng = np.random.default_rng(5)
    c = Case(6, [n + 120 for n in lens], heads, heads, d, ps, block, fmt, layout)
    start = np.array([(0, 7, 16, 100, 33)[b % 5] for b in range(len(lens))], dtype=np.int32)
    if len(lens) > 4:
        start[3] = -1                                               # an inactive row
    off = 1 + np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    total = int(off[-1]) + 2                                        # one token in front and two behind belong to no row
    k, v = bits(rng, total, heads, d, scale=0.5), bits(rng, total, heads, d, scale=3.0)
    if specials:
        k, v = with_specials(rng, k), with_specials(rng, v)
    cache = c.upload(rt)
    args = dev(c.table), dev(start), dev(off)
    cache.store(dev(k), dev(v), *args)
    kb, vb = cache.load(*args, total)
    torch.cuda.synchronize()
    assert int(cache.status_flag) == 0
    want = [np.zeros((total, heads, d)) for _ in range(2)]
    for b, n in enumerate(lens):
        if start[b] < 0 or n == 0:
            continue
        for side, x in enumerate((k, v)):
            c.cache.store(x[off[b]:off[b + 1]], side, c.table[b], int(start[b]))
            want[side][off[b]:off[b + 1]] = c.cache.read(side, c.table[b], start[b] + np.arange(n))
    c.same(cache)
    for got, ref in ((kb, want[0]), (vb, want[1])):
        got = f64(got)
        assert np.array_equal(np.isnan(got), np.isnan(ref))
        assert np.array_equal(got[~np.isnan(ref)], O.bf16_to_f64(O.f64_to_bf16_rne(ref))[~np.isnan(ref)])      # one rounding
    cache.store(dev(k), dev(v), *args)                              # the same again changes nothing
    c.same(cache)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("kind", ["normal", "ranges", "integers", "borders"])
def test_store_decides_every_code_as_the_definition_does(rt, fmt, kind):
    # many blocks: of every magnitude, of small integers (many values at a tie), largest values at and beside M 2^e
    import torch
    rng = np.random.default_rng(11)
    T, H, d, ps = 2000, 4, 64, 16
    x = rng.standard_normal((T, H, d))
    if kind == "ranges":
        x = np.ldexp(x, rng.integers(-140, 127, (T // ps, H, 1)).repeat(ps, 0))
    elif kind == "integers":
        x = np.rint(x * rng.integers(1, 40, (T, H, 1))) * np.ldexp(1.0, rng.integers(-20, 20, (T // ps, H, 1)).repeat(ps, 0))
    elif kind == "borders":
        x = np.clip(x, -4, 4)
        top = rng.choice([127, 127.5, 126.5, 255, 254, 448, 446, 450, 512, 1], (T, H)) * 2.0 ** rng.integers(-3, 4, (T, H))
        x[..., 0] = np.where(rng.random((T, H)) < 0.1, top, x[..., 0])
    x = O.f64_to_bf16_rne(x)
    kind_ = torch.int8 if fmt == Q.INT8 else torch.float8_e4m3fn
    cache = rt.Q8Cache.empty(T // ps, ps, H, d, 16, kind_)
    table = np.arange(T // ps, dtype=np.int32)[None]
    cache.store(dev(x), dev(x), dev(table), dev(np.zeros(1, np.int32)), dev(np.array([0, T], np.int32)))
    torch.cuda.synchronize()
    y = O.bf16_to_f64(x).reshape(T // ps, ps, H, d)
    need = np.array([[Q.needed(y[i, :, h], fmt) for h in range(H)] for i in range(T // ps)])
    codes = Q.encode(y / need[:, None, :, None], fmt)
    for side, pool in enumerate((cache.k_codes, cache.v_codes)):
        assert np.array_equal(host(cache.scales)[:, :, 0, side], need)
        got = host(pool)
        at = np.argwhere(got != codes)
        assert not len(at), (len(at), at[:3].tolist(), got[tuple(at[0])], codes[tuple(at[0])])


def test_store_beyond_the_table_and_bad_pages(rt):
    import torch
    from paper_2606_07665_b200 import binding as ac
    c = Case(8, [40, 40], 2, 2, 64, 16, 16, Q.INT8)
    cache = c.upload(rt)
    rng = np.random.default_rng(1)
    n = 16 * c.table.shape[1] + 3                                   # row 0 runs over its table row, row 1 into an unused entry
    x = bits(rng, 2 * n, 2, 64)
    off = np.array([0, n, 2 * n], dtype=np.int32)
    args = dev(c.table), dev(np.zeros(2, np.int32)), dev(off)
    cache.store(dev(x), dev(x), *args)
    kb, _ = cache.load(*args, 2 * n)
    torch.cuda.synchronize()
    assert int(cache.status_flag) == ac.AC_FLAG_PAGE_OOB | ac.AC_FLAG_POSITION_OOB
    for b in range(2):
        for side in range(2):
            c.cache.store(x[b * n:b * n + 48], side, c.table[b], 0)
    c.same(cache)
    assert not f64(kb).reshape(2, n, 2, 64)[:, 48:].any()           # tokens without a slot read as 0


def rotated(q, k, lens, variant, w, cos, sin, d):
    q_rot, k_rot = q.copy(), np.zeros_like(k)
    R = variant.get("rotary_dim", d)
    for b, n in enumerate(lens):
        if n < 0:
            continue
        for src, dst, wt in ((q, q_rot, w[0]), (k, k_rot, w[1])):
            for h in range(src.shape[1]):
                x = src[b, h] if wt is None else O.rms_norm_bf16(src[b, h], wt, 1e-5)
                dst[b, h] = O.rope_rotate_variant_bf16(x, cos[n], sin[n], R, variant.get("interleaved", False))
    return q_rot, k_rot


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d,ps,block", [(128, 16, 16), (64, 32, 32), (128, 96, 48), (64, 256, 256)])
@pytest.mark.parametrize("variant", [{}, dict(rotary_dim=34), dict(interleaved=True), dict(norm=True, interleaved=True, rotary_dim=32)])
def test_append(rt, fmt, d, ps, block, variant):
    """Token after token: blocks are begun, gone on with, outgrown by larger tokens, and every code follows."""
    import torch
    layout = "head_major" if variant else "token_major"
    lens = [0, 15, 16, -1, 100, 47]
    steps = 5
    c = Case(9, lens, 6, 3, d, ps, block, fmt, layout, room=steps)
    rng = np.random.default_rng(2)
    variant = dict(variant)
    norm = variant.pop("norm", False)
    cos, sin = W.rope_table(101 + steps, variant.get("rotary_dim", d), 10000.0)
    w = (bits(rng, d), bits(rng, d)) if norm else (None, None)
    cache, dlens = c.upload(rt), dev(c.lens)
    h = rt.Q8DecodeStep(cache, dev(c.table), dlens, 6, max_context_len=200, rope_cos=dev(cos), rope_sin=dev(sin),
                        rope_variants=dict(variant, q_norm_weight=None if w[0] is None else dev(w[0]),
                                           k_norm_weight=None if w[1] is None else dev(w[1]), norm_eps=1e-5))
    for step in range(steps):
        grow = 1.0 if norm else 2.0 ** rng.integers(-3, 4)
        q, k, v = bits(rng, 6, 6, d), bits(rng, 6, 3, d, scale=grow), bits(rng, 6, 3, d, scale=2.0 * grow)
        if step == 3:
            v[1, 0, 3], v[4, 1] = 0x7F80, 0                        # an infinity; a vector of zeros
        q_rot, k_rot = rotated(q, k, c.lens, variant, w, cos, sin, d)
        q_out = dev(q).clone()
        h.append(dev(q), dev(k), dev(v), q_out=q_out)
        torch.cuda.synchronize()
        assert int(h.status_flag) == 0
        assert np.array_equal(host(q_out), q_rot)
        for b, n in enumerate(c.lens):
            for side, x in enumerate((k_rot, v)):
                if n >= 0:
                    c.cache.store(x[b:b + 1], side, c.table[b], int(n))
        c.same(cache)
        c.lens[c.lens >= 0] += 1
        dlens.copy_(dev(c.lens))


def test_append_out_of_range(rt):
    import torch
    from paper_2606_07665_b200 import binding as ac
    c = Case(10, [3, 20, 5], 2, 2, 64, 16, 16, Q.E4M3)
    c.lens[:] = [16 * c.table.shape[1], 31, 33]                     # past the table row; a good one; an entry with no page
    c.table[2, 2] = c.num_pages
    cos, sin = W.rope_table(200, 64, 10000.0)
    cache = c.upload(rt)
    h = rt.Q8DecodeStep(cache, dev(c.table), dev(c.lens), 2, lens_host=c.lens, rope_cos=dev(cos), rope_sin=dev(sin))
    rng = np.random.default_rng(3)
    h.append(*[dev(bits(rng, 3, 2, 64)) for _ in range(3)])
    torch.cuda.synchronize()
    assert int(h.status_flag) == ac.AC_FLAG_PAGE_OOB | ac.AC_FLAG_POSITION_OOB
    pg = c.table[1, 1]
    other = np.arange(c.num_pages) != pg
    assert np.array_equal(host(cache.k_codes)[other], c.cache.pools[0][other])
    assert np.array_equal(host(cache.scales)[other], c.cache.scales[other], equal_nan=True)


def test_a_held_scale_that_is_no_number_of_the_library(rt):
    """A block that claims tokens under a zero, negative or infinite scale, or one that is no power of two."""
    import torch
    c = Case(12, [5, 5, 5, 5], 1, 1, 64, 16, 16, Q.INT8)
    for b, s in enumerate((0.0, -1.0, np.inf, 3.0)):
        c.cache.scales[c.table[b, 0], :, :, :] = s
    cache = c.upload(rt)
    rng = np.random.default_rng(4)
    v = bits(rng, 4, 1, 64)
    v[3] = W.f32_to_bf16_bits(np.full((1, 64), 21.0, np.float32))
    off = dev(np.arange(5, dtype=np.int32))
    cache.store(dev(v), dev(v), dev(c.table), dev(c.lens), off)
    torch.cuda.synchronize()
    s = host(cache.scales)[c.table[:, 0], 0, 0, 1]
    assert np.isfinite(s[0]) and np.isnan(s[1]) and np.isnan(s[2]) and s[3] == 3.0
    assert not host(cache.v_codes)[c.table[0, 0], :5].any()         # what was held under the scale 0
    assert (host(cache.v_codes)[c.table[3, 0], 5] == 7).all()       # 21 / 3


# ---- attention ---------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("Hq,Hkv,ps,block,layout", [(8, 2, 16, 16, "token_major"), (3, 3, 48, 48, "head_major"), (32, 2, 32, 16, "token_major"),
                                                    (9, 1, 256, 128, "head_major"), (14, 2, 64, 64, "head_major"), (1, 1, 80, 16, "token_major")])
@pytest.mark.parametrize("splits", [1, 3])
def test_attention(rt, fmt, d, Hq, Hkv, ps, block, layout, splits):
    c = Case(20 + splits, [0, 1, 15, 16, 31, 32, 200, -1, 777], Hq, Hkv, d, ps, block, fmt, layout)
    run_attention(rt, c, splits=splits)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (7, 4), (16, 16), (33, 100), (100, 5), (300, 64), (5000, 3), (64, 2**31 - 1),
                                          (2**31 - 1, 5), (150, 470), (150, 490)])
@pytest.mark.parametrize("splits", [1, 2, 5])
@pytest.mark.parametrize("d,ps,block", [(128, 16, 16), (64, 80, 16), (128, 64, 32)])
def test_attention_window_and_sinks(rt, fmt, window, sinks, splits, d, ps, block):
    c = Case(30, [0, 5, 100, 640, -1, 627], 8, 2, d, ps, block, fmt)
    for b, n in enumerate(c.lens):                                  # what is not attended is poisoned: neither read nor weighted
        seen = set(A.visible(int(n) + 1, window, sinks).tolist())
        for t in range(int(n) + 1):
            if t not in seen:
                for pool in c.cache.pools:
                    pool[c.table[b, t // ps], t % ps] = 0x7F
            if t % block == 0 and not seen & set(range(t, t + block)):
                c.cache.scales[c.table[b, t // ps], :, t % ps // block] = np.nan
    run_attention(rt, c, window=window, sinks=sinks, splits=splits)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("splits", [None, 4])
def test_attention_long_rows(rt, fmt, splits):
    c = Case(40, [9000, 4095], 8, 2, 128, 16, 16, fmt)
    run_attention(rt, c, splits=splits)


@pytest.mark.parametrize("Hq", [4, 12])
@pytest.mark.parametrize("splits", [1, 7, 700])
def test_attention_of_equal_weights_does_not_drift(rt, Hq, splits):
    """With q = 0 every weight is exactly 1 and, times a power of two, exact in fp16, so only the sums err.  Running sums
    of n terms of one sign are off by at most n 2^-24 of themselves; a warp of the widest launch has at most 1024 tiles: 2^-14.
    A tile's two steps on the tensor pipe lose at most 2^-22 each.  Joining 12 warps, 8 lanes and the splits: fewer than
    800 * 2^-24 < 2^-14.  Together below 2^-12 of the sum of positive values; the result's own rounding is 2^-8."""
    import torch
    c = Case(31, [131071], Hq, 1, 64, 32, 32, Q.INT8)
    for pool in c.cache.pools:
        pool &= 0x7F                                                # codes that are never negative
    h = rt.Q8DecodeStep(c.upload(rt), dev(c.table), dev(c.lens), c.Hq, lens_host=c.lens, num_splits=splits)
    out = h.attention(dev(np.zeros((1, Hq, 64), dtype=np.uint16)))
    torch.cuda.synchronize()
    V = c.cache.read(1, c.table[0], np.arange(131072), 0)
    ref = V.mean(0)
    assert (np.abs(f64(out)[0] - ref) <= (2.0**-8 * (1 + 2.0**-8) + 2.0**-12) * ref).all()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("q_scale", [8.0, 2.0**-120, 2.0**100])
def test_attention_peaked_and_scaled_queries(rt, fmt, q_scale):
    """Weights from 1 to nothing; queries of every magnitude (the softmax scale takes theirs back)."""
    c = Case(33, [300, 65], 8, 2, 128, 16, 16, fmt)
    scale = 0.0 if q_scale == 8.0 else 128.0**-0.5 / q_scale
    import torch
    q = bits(c.rng, c.B, c.Hq, c.d, scale=q_scale)
    if scale and scale < 2.0**-100 or scale > 2.0**100:
        scale = float(np.float32(scale))
    h = rt.Q8DecodeStep(c.upload(rt), dev(c.table), dev(c.lens), c.Hq, lens_host=c.lens, softmax_scale=scale)
    out = h.attention(dev(q))
    torch.cuda.synchronize()
    ref, room = A.attention(q, c.fetch, c.lens + 1, c.Hkv, scale=scale or None, slack=True)
    # products of up to 256 powers of two: 2^-11 of each weight, twice, instead of 2^-14
    check(f64(out), ref, room * 4, "peaked", c.floor(c.lens + 1))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("up", [True, False])
def test_attention_blocks_of_very_different_scales(rt, fmt, up):
    """V's scales grow (or fall) by 2^6 from block to block, K's by 2: the largest block decides nearly all of the result, whatever
    came before it.  (Sums of |q k| of up to 256 powers of two: 2^-11 of each weight, twice, instead of 2^-14.)"""
    c = Case(34, [255], 8, 2, 128, 16, 16, fmt)
    for i in range(16):
        page = c.table[0, i]
        c.cache.scales[page, :, 0, 1] = 2.0 ** (6 * (i if up else 15 - i) - 45)
        c.cache.scales[page, :, 0, 0] = 2.0 ** ((i if up else 15 - i) - 16)
    run_attention(rt, c, splits=1, slack=4)
    run_attention(rt, c, splits=4, slack=4)


@pytest.mark.parametrize("fmt", FORMATS)
def test_attention_of_a_block_that_is_nan(rt, fmt):
    import torch
    c = Case(35, [100, 100, 100], 4, 2, 64, 16, 16, fmt)
    c.cache.scales[c.table[0, 2], 0, 0, 0] = np.nan                 # K of row 0, head 0
    c.cache.scales[c.table[1, 6], 1, 0, 1] = np.nan                 # V of row 1, head 1
    q = bits(c.rng, 3, 4, 64)
    h = rt.Q8DecodeStep(c.upload(rt), dev(c.table), dev(c.lens), 4, lens_host=c.lens)
    out = f64(h.attention(dev(q)))
    torch.cuda.synchronize()
    assert np.isnan(out[0, :2]).all() and np.isnan(out[1, 2:]).all()
    assert np.isfinite(out[0, 2:]).all() and np.isfinite(out[1, :2]).all() and np.isfinite(out[2]).all()


@pytest.mark.parametrize("ps", [16, 64])
def test_attention_bad_pages_read_as_zeros(rt, ps):
    import torch
    c = Case(36, [200], 4, 2, 64, ps, 16, Q.E4M3)
    q = bits(c.rng, 1, 4, 64)
    ref_case = Case(36, [200], 4, 2, 64, ps, 16, Q.E4M3)
    gone = c.table[0, 1]
    for pool in ref_case.cache.pools:
        pool[gone] = 0
    ref_case.cache.scales[gone] = 1.0
    ref, room = A.attention(q, ref_case.fetch, c.lens + 1, 2, slack=True)
    for bad in (-1, c.num_pages, 2**31 - 1, -2**31):
        c.table[0, 1] = bad
        h = rt.Q8DecodeStep(c.upload(rt), dev(c.table), dev(c.lens), 4, lens_host=c.lens)
        out = h.attention(dev(q))
        torch.cuda.synchronize()
        check(f64(out), ref, room, bad)


def test_attention_of_rows_that_outgrew_the_plan(rt):
    c = Case(37, [500, 700, 20], 8, 2, 128, 32, 32, Q.INT8)
    run_attention(rt, c, splits=3, max_context_len=100)
    run_attention(rt, c, splits=2, max_context_len=64, window=300, sinks=20)


def test_attention_over_the_cached_tokens_alone(rt):
    c = Case(38, [0, 1, 16, 33, -1], 8, 2, 64, 16, 16, Q.INT8, room=0)
    run_attention(rt, c, new_tokens=0)
    run_attention(rt, c, new_tokens=0, splits=2)


@pytest.mark.parametrize("B", [1, 70])
@pytest.mark.parametrize("row_order", ["auto", None])
def test_attention_many_rows(rt, B, row_order):
    rng = np.random.default_rng(B)
    c = Case(39, rng.integers(0, 600, B), 16, 8, 64, 32, 16, Q.E4M3)
    run_attention(rt, c, row_order=row_order)
