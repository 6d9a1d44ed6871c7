"""The 4-bit cache on the GPU against its oracle: what is written is compared code by code, attention within a bound
derived from its roundings."""
import numpy as np
import pytest

from oracle import paged_decode_oracle as O
from oracle import q4_cache_oracle as Q
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
    import torch
    if t.dtype == torch.bfloat16:
        t = t.view(torch.int16)
    a = t.cpu().numpy()
    return a.view(np.uint16) if a.dtype == np.int16 else a


def f64(t):
    return O.bf16_to_f64(host(t))


class Case:
    """A quantised cache of random values under a scattered block table, everything that no row holds poisoned."""

    def __init__(self, rt, seed, lens, Hq, Hkv, d, ps, group, layout="token_major", room=1, v_scale=1.0, k_scale=1.0, spare=3):
        rng = self.rng = np.random.default_rng(seed)
        self.lens = np.asarray(lens, dtype=np.int32)
        self.B, self.Hq, self.Hkv, self.d, self.ps, self.group, self.layout = len(lens), Hq, Hkv, d, ps, group, layout
        need = [-(-(max(int(n), 0) + room) // ps) for n in lens]
        self.num_pages = sum(need) + spare
        perm = rng.permutation(self.num_pages)
        self.table = np.full((self.B, max(need) + 1), -7, dtype=np.int32)      # unused entries name no page at all
        at = 0
        for b, k in enumerate(need):
            self.table[b, :k] = perm[at:at + k]
            at += k
        # [page, slot, head, ...] on the host, whatever the layout on the device
        self.k = rng.integers(0, 256, (self.num_pages, ps, Hkv, d // 2)).astype(np.uint8)
        self.v = rng.integers(0, 256, (self.num_pages, ps, Hkv, d // 2)).astype(np.uint8)
        G = d // group
        self.prm = np.full((self.num_pages, Hkv, ps, 2, G, 2), Q.NAN, dtype=np.uint16)
        for b in range(self.B):
            t = np.arange(max(int(lens[b]), 0) + (room if lens[b] >= 0 else 0))
            for i in t:
                pg, sl = self.table[b, i // ps], i % ps
                for side, sc in ((0, k_scale), (1, v_scale)):
                    s = sc * (0.15 + 0.1 * rng.random((Hkv, G)))
                    self.prm[pg, :, sl, side, :, 0] = W.f32_to_bf16_bits(s.astype(np.float32))
                    self.prm[pg, :, sl, side, :, 1] = W.f32_to_bf16_bits((-7.5 * s + 0.3 * sc * rng.standard_normal((Hkv, G))).astype(np.float32))

    def upload(self, rt):
        import torch
        move = (lambda x: x) if self.layout == "token_major" else (lambda x: x.transpose(0, 2, 1, 3))
        return rt.Q4Cache(dev(move(self.k)), dev(move(self.v)), dev(self.prm).view(torch.bfloat16), layout=self.layout)

    def download(self, c):
        move = (lambda x: x) if self.layout == "token_major" else (lambda x: x.transpose(0, 2, 1, 3))
        return move(host(c.k_codes)), move(host(c.v_codes)), host(c.params)

    def fetch(self, b, h, t):
        pg, sl = self.table[b, t // self.ps], t % self.ps
        kp, vp = self.prm[pg, h, sl, 0], self.prm[pg, h, sl, 1]
        K, _ = Q.values(self.k[pg, sl, h], kp[..., 0], kp[..., 1])
        V, cs = Q.values(self.v[pg, sl, h], vp[..., 0], vp[..., 1])
        return K, V, np.abs(cs) + np.abs(V) / 8


def check(got, ref, room, what):
    """Each weight times a V scale is rounded to fp16 (2^-11 relative) and multiplies |c s|; scores are fp32 sums of
    d products, whose error moves a weight by less than 2^-14 at these sizes (|c q| s sums below 100, 2^-22 each), and
    the fp32 accumulation of the weighted values adds as little: 2^-14 of |V| and of |c s|.  `room` is sum_t p_t (|c s| +
    |V| / 8), so 2^-11 of it covers 2^-11 |c s| + 2^-14 |V|.  The result is rounded to bf16, 2^-8 relative."""
    bound = 2.0**-8 * np.abs(ref) * (1 + 2.0**-8) + (2.0**-11 + 2.0**-14) * room + 1e-30
    err = np.abs(got - ref)
    assert np.isfinite(got).all(), what
    assert (err <= bound).all(), (what, float((err / bound).max()))
    return float((err / bound).max())


def run_attention(rt, c, window=0, sinks=0, splits=None, q=None, new_tokens=1, row_order="auto", q_scale=1.0):
    import torch
    q = bits(c.rng, c.B, c.Hq, c.d, scale=q_scale) if q is None else q
    cache = c.upload(rt)
    h = rt.Q4DecodeStep(cache, dev(c.table), dev(c.lens), c.Hq, lens_host=c.lens, window=window, sinks=sinks, num_splits=splits,
                        new_tokens=new_tokens, row_order=row_order)
    out = h.attention(dev(q))
    again = h.attention(dev(q))
    torch.cuda.synchronize()
    assert torch.equal(out, again), "two calls differ"
    n = np.where(c.lens >= 0, c.lens + new_tokens, 0)
    ref, room = Q.attention(q, c.fetch, n, c.Hkv, window, sinks, slack=True)
    worst = check(f64(out), ref, room, f"splits {h.num_splits}")
    assert not f64(out)[n <= 0].any()
    return worst, h, out


# ---- writing ---------------------------------------------------------------------------------------------------


def with_specials(rng, x):
    """Puts into the first heads: infinities, NaN, both zeros, a constant, subnormals, the type's extremes, ties."""
    x = x.copy()
    flat = x.reshape(-1, x.shape[-1])
    for i, vals in enumerate(([0x7F80], [0xFF80, 0x3F80], [0x7FC0], [0x0000, 0x8000], [0x4049], [0x0001, 0x8003, 0x0007],
                              [0x7F7F, 0xFF7F, 0x7E80, 0x0000], [0x4170, 0x3F00, 0x3FC0, 0x4020, 0x0000])):
        if i < len(flat):
            flat[i] = np.resize(np.array(vals, dtype=np.uint16), x.shape[-1])
            if i == 2:
                flat[i, 1:] = 0x3F80
    return x


@pytest.mark.parametrize("d,group", [(128, 128), (128, 64), (128, 32), (64, 64), (64, 32)])
@pytest.mark.parametrize("layout", ["token_major", "head_major"])
@pytest.mark.parametrize("total_heads,ps,lens", [(1, 16, [0]), (3, 32, [5, 0, 0, 33, 64]), (8, 48, [100, 1, 17]),
                                                  (40, 16, [3, 0, 18]), (1, 64, [700, 0, 331])])
def test_store_and_load(rt, d, group, layout, total_heads, ps, lens):
    import torch
    rng = np.random.default_rng(5)
    c = Case(rt, 6, [n + 20 for n in lens], total_heads, total_heads, d, ps, group, layout)
    start = np.array([(7 * b) % 20 for b in range(len(lens))], dtype=np.int32)
    if len(lens) > 3:
        start[3] = -1                                               # an inactive row
    off = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    total = int(off[-1]) + 2                                        # two tokens that belong to no row
    k, v = with_specials(rng, bits(rng, total, total_heads, d)), with_specials(rng, bits(rng, total, total_heads, d, scale=3.0))
    cache = c.upload(rt)
    cache.store(dev(k), dev(v), dev(c.table), dev(start), dev(off))
    kb, vb = cache.load(dev(c.table), dev(start), dev(off), total)
    torch.cuda.synchronize()
    assert int(cache.status_flag) == 0
    want_k, want_v = np.zeros((total, total_heads, d)), np.zeros((total, total_heads, d))
    for b, n in enumerate(lens):
        for i in range(n if start[b] >= 0 else 0):
            pg, sl, t = c.table[b, (start[b] + i) // ps], (start[b] + i) % ps, off[b] + i
            for side, (x, pool, want) in enumerate(((k, c.k, want_k), (v, c.v, want_v))):
                codes, s, m = Q.quantise(x[t], group)
                pool[pg, sl] = Q.pack(codes)
                c.prm[pg, :, sl, side] = np.stack([s, m], -1)
                want[t] = Q.values(Q.pack(codes), s, m)[0]
    gk, gv, gp = c.download(cache)
    for what, a, b in (("K codes", gk, c.k), ("V codes", gv, c.v), ("parameters", gp, c.prm)):
        at = np.argwhere(a != b)
        assert not len(at), (what, at[:4].tolist(), a[a != b][:8].tolist(), b[a != b][:8].tolist())
    for got, want in ((kb, want_k), (vb, want_v)):
        got = f64(got)
        assert np.array_equal(np.isnan(got), np.isnan(want))
        # one bf16 rounding (half a bf16 subnormal step at the bottom)
        assert (np.abs(got - want)[~np.isnan(want)] <= (2.0**-8 * (1 + 2.0**-8) * np.abs(want) + 2.0**-134)[~np.isnan(want)]).all()


@pytest.mark.parametrize("d,group", [(128, 64), (64, 32), (128, 128)])
@pytest.mark.parametrize("kind", ["normal", "ranges", "integers", "offset"])
def test_store_decides_every_code_as_the_definition_does(rt, d, group, kind):
    # many vectors: of every magnitude, of small integers (many quotients at a half), far from zero (few codes apart)
    import torch
    rng = np.random.default_rng(11)
    T, H, ps = 3000, 4, 64
    x = rng.standard_normal((T, H, d))
    if kind == "ranges":
        x = np.ldexp(x, rng.integers(-140, 127, (T, H, 1)))
    elif kind == "integers":
        x = np.rint(x * rng.integers(1, 40, (T, H, 1))) * np.ldexp(1.0, rng.integers(-20, 20, (T, H, 1)))
    elif kind == "offset":
        x = x + rng.integers(-200, 200, (T, H, 1))
    x = O.f64_to_bf16_rne(x)
    cache = rt.Q4Cache.empty(T // ps + 1, ps, H, d, group)
    table = np.arange(T // ps + 1, dtype=np.int32)[None]
    cache.store(dev(x), dev(x), dev(table), dev(np.zeros(1, np.int32)), dev(np.array([0, T], np.int32)))
    torch.cuda.synchronize()
    codes, s, m = Q.quantise(x, group)
    for side, pool in enumerate((cache.k_codes, cache.v_codes)):
        got = Q.unpack(host(pool).reshape(-1, H, d // 2)[:T])
        at = np.argwhere(got != codes)
        assert not len(at), (len(at), at[:3].tolist(), got[tuple(at[0])], codes[tuple(at[0])])
        p = host(cache.params)[:, :, :, side].transpose(0, 2, 1, 3, 4).reshape(-1, H, d // group, 2)[:T]
        assert np.array_equal(p[..., 0], s) and np.array_equal(p[..., 1], m)


def test_store_beyond_the_table_and_bad_pages(rt):
    import torch
    from paper_2606_07665_b200 import binding as ac
    c = Case(rt, 8, [40, 40], 2, 2, 64, 16, 32)
    cache = c.upload(rt)
    rng = np.random.default_rng(1)
    n = 16 * c.table.shape[1] + 3                                   # row 0 runs over its table row, row 1 into an unused entry
    x = dev(bits(rng, 2 * n, 2, 64))
    off = dev(np.array([0, n, 2 * n], dtype=np.int32))
    before = c.download(cache)
    cache.store(x, x, dev(c.table), dev(np.zeros(2, np.int32)), off)
    kb, _ = cache.load(dev(c.table), dev(np.zeros(2, np.int32)), off, 2 * n)
    torch.cuda.synchronize()
    assert int(cache.status_flag) == ac.AC_FLAG_PAGE_OOB | ac.AC_FLAG_POSITION_OOB
    after = c.download(cache)
    untouched = np.setdiff1d(np.arange(c.num_pages), c.table[c.table >= 0])
    for a, b in zip(before, after):
        assert np.array_equal(a[untouched], b[untouched])
    assert not f64(kb).reshape(2, n, 2, 64)[:, 48:].any()           # tokens without a slot read as 0


@pytest.mark.parametrize("d,group", [(128, 128), (128, 64), (128, 32), (64, 64), (64, 32)])
@pytest.mark.parametrize("variant", [{}, dict(rotary_dim=32), dict(interleaved=True), dict(norm=True, interleaved=True)])
def test_append(rt, d, group, variant):
    import torch
    layout = "head_major" if variant else "token_major"
    c = Case(rt, 9, [0, 15, 16, -1, 100], 6, 3, d, 16, group, layout)
    rng = np.random.default_rng(2)
    q, k, v = bits(rng, 5, 6, d), with_specials(rng, bits(rng, 5, 3, d)), with_specials(rng, bits(rng, 5, 3, d))
    k[:3] = bits(rng, 3, 3, d) if variant else k[:3]                # the norm and the rotation of NaN are not at stake
    variant = dict(variant)
    norm = variant.pop("norm", False)
    R = variant.get("rotary_dim", d)
    cos, sin = W.rope_table(101, R, 10000.0)
    w = (bits(rng, d), bits(rng, d)) if norm else (None, None)
    q_rot, k_rot = q.copy(), np.zeros_like(k)
    for b, n in enumerate(c.lens):
        if n < 0:
            continue
        for src, dst, wt in ((q, q_rot, w[0]), (k, k_rot, w[1])):
            for h in range(src.shape[1]):
                x = src[b, h] if wt is None else O.rms_norm_bf16(src[b, h], wt, 1e-5)
                dst[b, h] = O.rope_rotate_variant_bf16(x, cos[n], sin[n], R, variant.get("interleaved", False))
    cache = c.upload(rt)
    h = rt.Q4DecodeStep(cache, dev(c.table), dev(c.lens), 6, lens_host=c.lens, rope_cos=dev(cos), rope_sin=dev(sin),
                        rope_variants=dict(variant, q_norm_weight=None if w[0] is None else dev(w[0]),
                                           k_norm_weight=None if w[1] is None else dev(w[1]), norm_eps=1e-5))
    q_out = dev(q).clone()
    h.append(dev(q), dev(k), dev(v), q_out=q_out)
    torch.cuda.synchronize()
    assert int(h.status_flag) == 0
    assert np.array_equal(host(q_out), q_rot)
    for b, n in enumerate(c.lens):
        if n < 0:
            continue
        pg, sl = c.table[b, n // 16], n % 16
        for side, (x, pool) in enumerate(((k_rot, c.k), (v, c.v))):
            codes, s, m = Q.quantise(x[b], group)
            pool[pg, sl] = Q.pack(codes)
            c.prm[pg, :, sl, side] = np.stack([s, m], -1)
    gk, gv, gp = c.download(cache)
    assert np.array_equal(gk, c.k) and np.array_equal(gv, c.v) and np.array_equal(gp, c.prm)


def test_append_out_of_range(rt):
    import torch
    from paper_2606_07665_b200 import binding as ac
    c = Case(rt, 10, [3, 20, 5], 2, 2, 64, 16, 64)
    c.lens[:] = [16 * c.table.shape[1], 31, 33]                     # past the table row; a good one; an entry with no page
    c.table[2, 2] = c.num_pages
    cos, sin = W.rope_table(200, 64, 10000.0)
    cache = c.upload(rt)
    h = rt.Q4DecodeStep(cache, dev(c.table), dev(c.lens), 2, lens_host=c.lens, rope_cos=dev(cos), rope_sin=dev(sin))
    rng = np.random.default_rng(3)
    h.append(*[dev(bits(rng, 3, 2, 64)) for _ in range(3)])
    torch.cuda.synchronize()
    assert int(h.status_flag) == ac.AC_FLAG_PAGE_OOB | ac.AC_FLAG_POSITION_OOB
    gk, gv, gp = c.download(cache)
    pg, sl = c.table[1, 1], 15
    changed = np.zeros(gk.shape[:2], dtype=bool)
    changed[pg, sl] = True
    assert np.array_equal(gk[~changed], c.k[~changed]) and np.array_equal(gv[~changed], c.v[~changed])


# ---- attention ---------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("d,group", [(128, 128), (128, 64), (128, 32), (64, 64), (64, 32)])
@pytest.mark.parametrize("Hq,Hkv,ps,layout", [(8, 2, 16, "token_major"), (3, 3, 48, "head_major"), (32, 2, 32, "token_major"),
                                              (9, 1, 256, "head_major"), (14, 2, 16, "head_major")])
@pytest.mark.parametrize("splits", [1, 3])
def test_attention(rt, d, group, Hq, Hkv, ps, layout, splits):
    c = Case(rt, 20 + splits, [0, 1, 15, 16, 31, 32, 200, -1, 777], Hq, Hkv, d, ps, group, layout)
    run_attention(rt, c, splits=splits)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (7, 4), (16, 16), (33, 100), (100, 5), (300, 64), (5000, 3), (64, 2**31 - 1),
                                          (2**31 - 1, 5), (150, 470), (150, 490)])
@pytest.mark.parametrize("splits", [1, 2, 5])
@pytest.mark.parametrize("d,ps", [(128, 16), (64, 80)])
def test_attention_window_and_sinks(rt, window, sinks, splits, d, ps):
    c = Case(rt, 30, [0, 5, 100, 640, -1, 627], 8, 2, d, ps, 32)
    for b, n in enumerate(c.lens):                                  # what is not attended is poisoned: neither read nor weighted
        seen = set(Q.visible(int(n) + 1, window, sinks).tolist())
        for t in range(int(n) + 1):
            if t not in seen:
                c.prm[c.table[b, t // ps], :, t % ps] = Q.NAN
    run_attention(rt, c, window=window, sinks=sinks, splits=splits)


@pytest.mark.parametrize("splits", [None, 4])
def test_attention_long_rows(rt, splits):
    c = Case(rt, 40, [9000, 4095], 8, 2, 128, 16, 64)
    run_attention(rt, c, splits=splits)


@pytest.mark.parametrize("Hq", [4, 12])
@pytest.mark.parametrize("splits", [1, 7])
def test_attention_of_equal_weights_does_not_drift(rt, Hq, splits):
    """With q = 0 every weight is exactly 1 and a weight times a scale (8 bits times a power of two) exact in fp16, so
    only the sums err.  Twelve warps share the row in the widest launch, eight in that of more than eight heads: at most
    512 tiles a warp.  Running sums of n terms of one sign are off by at most n 2^-24 of themselves; there are two (the
    codes and the minima, |m| below 8 s, as large as |c s| on average): 2 * 512 * 2^-24 = 2^-14.  A tile's two steps on
    the tensor pipe lose at most 2^-22 each of a byte sum that is 17 times the even code's: 2^-17.  Joining 12 warps, 8
    lanes and 7 splits: 27 * 2^-24.  Together below 2^-13 of sum_t p_t |c s|; the result's own rounding is 2^-8."""
    import torch
    c = Case(rt, 31, [131071], Hq, 1, 64, 32, 64)
    h = rt.Q4DecodeStep(c.upload(rt), dev(c.table), dev(c.lens), c.Hq, lens_host=c.lens, num_splits=splits)
    q = np.zeros((1, Hq, 64), dtype=np.uint16)
    out = f64(h.attention(dev(q)))
    torch.cuda.synchronize()
    ref, room = Q.attention(q, c.fetch, c.lens + 1, 1, 0, 0, slack=True)
    assert (np.abs(out - ref) <= 2.0**-8 * np.abs(ref) + 2.0**-13 * room).all(), float((np.abs(out - ref) / room).max())


@pytest.mark.parametrize("new_tokens", [0, 1])
def test_attention_new_tokens_and_plan(rt, new_tokens):
    c = Case(rt, 41, [0, 64, 1500, -1], 16, 4, 128, 16, 64)
    run_attention(rt, c, new_tokens=new_tokens)


@pytest.mark.parametrize("lens,Hq,Hkv,splits", [
    ([40000], 4, 1, None), ([300 + 37 * i for i in range(60)], 8, 4, None), ([(i * 7) % 70 - 1 for i in range(700)], 6, 3, 2),
    ([100, 3000], 4, 2, 47),                                # as many splits as fit; most of the short row's are empty
    ([2000] * 40, 64, 4, None),                             # sixteen heads, more than one CTA per SM
    ([500 + i for i in range(120)], 16, 4, 1)])             # four-warp CTAs
def test_attention_launch_shapes(rt, lens, Hq, Hkv, splits):
    run_attention(rt, Case(rt, 49, lens, Hq, Hkv, 64, 16, 32), splits=splits)


def test_attention_two_objects_on_two_streams(rt):
    # each object has its workspace, so their calls may overlap
    import torch
    c = Case(rt, 48, [5000, 100, 3000], 8, 2, 128, 16, 64)
    cache, q = c.upload(rt), dev(bits(c.rng, 3, 8, 128))
    table, lens = dev(c.table), dev(c.lens)
    objects = [rt.Q4DecodeStep(cache, table, lens, 8, lens_host=c.lens, num_splits=5) for _ in range(2)]
    want = objects[0].attention(q)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [[torch.empty_like(q) for _ in range(30)] for _ in range(2)]
    for i in range(30):
        for h, st, o in zip(objects, streams, outs):
            h.attention(q, out=o[i], stream=st)
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for os in outs for o in os)


@pytest.mark.parametrize("handle", [False, True])
def test_results_belong_to_the_stream_that_writes_them(rt, handle):
    """Memory of a result (and of the step's rotated queries, which nobody holds) that is dropped while another stream still
    writes it must not go to the current stream's next tensor."""
    import torch
    c = Case(rt, 41, [700, 300], 8, 2, 64, 16, 64)
    cache = c.upload(rt)
    cos, sin = W.rope_table(1024, 64, 10000.0)
    h = rt.Q4DecodeStep(cache, dev(c.table), dev(c.lens), 8, lens_host=c.lens, rope_cos=dev(cos), rope_sin=dev(sin))
    q, k, v = (dev(bits(c.rng, 2, n, 64)).view(torch.bfloat16) for n in (8, 2, 2))
    start, off = dev(np.zeros(2, dtype=np.int32)), dev(np.array([0, 4, 8], dtype=np.int32))
    want = h.step(q, k, v)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    stream = side.cuda_stream if handle else side
    made = []
    own = h._new
    h._new = cache._new = lambda *a: made.append(own(*a)) or made[-1]
    got = h.step(q, k, v, stream=stream)
    cache.load(dev(c.table), start, off, 8, stream=stream)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and len(made) == 4
    where = {t.data_ptr() for t in made}
    shapes = [t.shape for t in made]
    del made, got
    assert not where & {t.data_ptr() for t in [torch.empty(s, dtype=torch.bfloat16, device="cuda") for s in shapes]}


def test_append_in_place_rotates_the_queries_where_they_are(rt):
    import torch
    c = Case(rt, 50, [5, 40], 4, 2, 128, 16, 64)
    cos, sin = W.rope_table(64, 128, 10000.0)
    h = rt.Q4DecodeStep(c.upload(rt), dev(c.table), dev(c.lens), 4, lens_host=c.lens, rope_cos=dev(cos), rope_sin=dev(sin))
    q, k, v = (dev(bits(c.rng, 2, n, 128)) for n in (4, 2, 2))
    want = h.append(q, k, v).clone()
    h.append(q, k, v, q_out=q)
    torch.cuda.synchronize()
    assert torch.equal(q, want)


def test_attention_row_order(rt):
    c = Case(rt, 42, [10, 500, 200, 700], 8, 2, 128, 16, 64)
    a = run_attention(rt, c, q=(q := bits(c.rng, 4, 8, 128)))[2]
    b = run_attention(rt, c, q=q, row_order=[3, 1, 2, 0])[2]
    assert np.array_equal(host(a), host(b))


@pytest.mark.parametrize("kind", ["rising", "falling", "peaks", "v_rising", "v_falling", "v_tiny", "v_huge", "v_zero_first", "q_tiny", "q_zero"])
def test_attention_references_follow(rt, kind):
    # the softmax reference and the power of two on V's scales have to follow whatever comes, in either order
    c = Case(rt, 43, [800, 63], 8, 2, 128, 16, 64, v_scale=dict(v_tiny=2.0**-100, v_huge=2.0**100).get(kind, 1.0))
    q = bits(c.rng, 2, 8, 128)
    q[:, :, :] = W.f32_to_bf16_bits(np.abs(W.bf16_bits_to_f32(q)))
    if kind == "q_tiny":
        q = W.f32_to_bf16_bits(W.bf16_bits_to_f32(q) * np.float32(2.0**-110))
    if kind == "q_zero":
        q[:] = 0
        q[:, 1] = 0x8000
    for b, n in enumerate(c.lens):
        for t in range(int(n) + 1):
            at = c.table[b, t // 16], slice(None), t % 16
            x = t / 800
            if kind in ("rising", "falling"):                       # the minimum moves the score: about 100 powers of two over the row
                y = (x if kind == "rising" else 1 - x) * 8
                c.prm[at + (0, slice(None), 1)] = W.f32_to_bf16_bits(np.full((2, 2), y, np.float32))
            elif kind == "peaks" and t % 97 == 13:
                c.prm[at + (0, slice(None), 1)] = W.f32_to_bf16_bits(np.full((2, 2), 0.3 * (t // 97), np.float32))
            elif kind in ("v_rising", "v_falling"):
                e = int((x if kind == "v_rising" else 1 - x) * 60 - 30)
                for i in (0, 1):
                    w = W.bf16_bits_to_f32(c.prm[at + (1, slice(None), i)]) * np.float32(2.0**e)
                    c.prm[at + (1, slice(None), i)] = W.f32_to_bf16_bits(w)
            elif kind == "v_zero_first" and t < 700:
                c.prm[at + (1, slice(None), 0)] = 0
    run_attention(rt, c, q=q)
    run_attention(rt, c, q=q, splits=3)


def test_attention_poison_of_one_row_stays_there(rt):
    # a NaN inside a row's tokens makes that row's group NaN and no other row
    import torch
    c = Case(rt, 44, [100, 100], 4, 2, 64, 16, 32)
    c.prm[c.table[0, 2], 1, 3, 1, 0, 1] = Q.NAN                     # row 0, head 1, token 35, V, first group
    cache = c.upload(rt)
    h = rt.Q4DecodeStep(cache, dev(c.table), dev(c.lens), 4, lens_host=c.lens)
    q = bits(c.rng, 2, 4, 64)
    out = f64(h.attention(dev(q)))
    torch.cuda.synchronize()
    bad = np.zeros((2, 4, 64), dtype=bool)
    bad[0, 2:, :32] = True
    assert np.array_equal(np.isnan(out), bad)


def test_attention_pages_outside_the_pool_read_as_zeros(rt):
    import torch
    c = Case(rt, 45, [47], 4, 2, 64, 16, 32)
    good = c.table.copy()
    c.table[0, 1] = c.num_pages + 5
    cache = c.upload(rt)
    h = rt.Q4DecodeStep(cache, dev(c.table), dev(c.lens), 4, lens_host=c.lens)
    q = bits(c.rng, 1, 4, 64)
    out = h.attention(dev(q))
    torch.cuda.synchronize()
    c.table = good
    pg = good[0, 1]
    c.k[pg], c.v[pg], c.prm[pg] = 0, 0, 0
    ref, room = Q.attention(q, c.fetch, [48], 2, slack=True)
    check(f64(out), ref, room, "zeros")


# ---- a run of steps ------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("window,sinks,splits", [(0, 0, 1), (0, 0, 2), (40, 6, 2)])
def test_store_then_captured_steps(rt, window, sinks, splits):
    # a prompt is stored, then steps are replayed from one captured graph with new lengths and inputs, on another stream
    import torch
    rng = np.random.default_rng(7)
    B, Hq, Hkv, d, ps, group, steps = 3, 8, 2, 128, 16, 64, 20
    lens = np.array([50, 0, 131], dtype=np.int32)
    c = Case(rt, 46, lens, Hq, Hkv, d, ps, group, room=steps)
    cache = rt.Q4Cache.empty(c.num_pages, ps, Hkv, d, group)
    off = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    k, v = bits(rng, int(off[-1]), Hkv, d), bits(rng, int(off[-1]), Hkv, d)
    cos, sin = W.rope_table(200, d, 10000.0)
    table, lens_d = dev(c.table), dev(lens)
    cache.store(dev(k), dev(v), table, dev(np.zeros(B, np.int32)), dev(off))
    c.prm[:] = Q.NAN
    for b in range(B):
        for t in range(lens[b]):
            write(c, b, t, k[off[b] + t], v[off[b] + t])
    h = rt.Q4DecodeStep(cache, table, lens_d, Hq, max_context_len=160, window=window, sinks=sinks, num_splits=splits,
                        rope_cos=dev(cos), rope_sin=dev(sin))
    q_in, k_new, v_new = (dev(np.zeros((B, n, d), np.uint16)) for n in (Hq, Hkv, Hkv))
    q_rot, out = torch.empty_like(q_in), torch.empty_like(q_in)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        h.step(q_in, k_new, v_new, q_rot=q_rot, out=out)
    for i in range(steps):
        q, kn, vn = bits(rng, B, Hq, d), bits(rng, B, Hkv, d), bits(rng, B, Hkv, d)
        q_in.copy_(dev(q)), k_new.copy_(dev(kn)), v_new.copy_(dev(vn))
        lens_d.copy_(dev((lens + i).astype(np.int32)))
        graph.replay()
        torch.cuda.synchronize()
        qr = np.zeros_like(q)
        for b in range(B):
            p = lens[b] + i
            for hh in range(Hq):
                qr[b, hh] = O.rope_rotate_bf16(q[b, hh], cos[p], sin[p])
            write(c, b, p, np.stack([O.rope_rotate_bf16(kn[b, hh], cos[p], sin[p]) for hh in range(Hkv)]), vn[b])
        ref, room = Q.attention(qr, c.fetch, lens + i + 1, Hkv, window, sinks, slack=True)
        check(f64(out), ref, room, f"step {i}")
    gk, gv, gp = c.download(cache)
    held = [(c.table[b, t // ps], t % ps) for b in range(B) for t in range(lens[b] + steps)]
    pg, sl = np.array(held).T
    assert np.array_equal(gk[pg, sl], c.k[pg, sl]) and np.array_equal(gv[pg, sl], c.v[pg, sl])
    assert np.array_equal(gp[pg, :, sl], c.prm[pg, :, sl])


def write(c, b, t, k, v):
    pg, sl = c.table[b, t // c.ps], t % c.ps
    for side, (x, pool) in enumerate(((k, c.k), (v, c.v))):
        codes, s, m = Q.quantise(x, c.group)
        pool[pg, sl] = Q.pack(codes)
        c.prm[pg, :, sl, side] = np.stack([s, m], -1)


def test_runner_refusals(rt):
    import torch
    c = Case(rt, 47, [10, 20], 4, 2, 64, 16, 32)
    cache = c.upload(rt)
    h = rt.Q4DecodeStep(cache, dev(c.table), dev(c.lens), 4, lens_host=c.lens)
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16, device="cuda")
    for bad in (q.float(), q[:1], q.transpose(0, 1).contiguous().transpose(0, 1), q.cpu()):
        with pytest.raises(ValueError):
            h.attention(bad)
    with pytest.raises(ValueError, match="rope"):
        h.append(q, q[:, :2].contiguous(), q[:, :2].contiguous())
    with pytest.raises(ValueError):
        rt.Q4DecodeStep(cache, dev(c.table), dev(c.lens[:1]), 4)
    with pytest.raises(ValueError):
        rt.Q4DecodeStep(cache, dev(c.table), dev(c.lens), 5)
    with pytest.raises(ValueError):
        rt.Q4Cache(cache.k_codes, cache.v_codes[:2], cache.params)
    with pytest.raises(ValueError):
        cache.store(q, q, dev(c.table), dev(c.lens), dev(np.zeros(3, np.int32)))       # four heads for two
