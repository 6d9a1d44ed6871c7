"""Refusals of the 8-bit cache's and the rotary entry points: decided on the host, before any device is touched."""
import ctypes

import pytest

NULL, SHAPE, UNSUPPORTED, ALIGN, WORKSPACE = 1, 2, 3, 4, 5
P = 1 << 20                                       # a pointer that is never followed
SHAPE6 = (1, 8, 2, 64, 32, 64)                    # B, Hq, Hkv, d, page_size, num_pages


@pytest.fixture(scope="module")
def ac():
    from paper_2606_07665_b200 import binding, build
    build.build()
    return binding


def cache(ac, **kw):
    f = dict(k_codes=P, v_codes=P, scales=P, stride_page=32 * 2 * 64, stride_token=128, stride_head=64, stride_scales=8, block=16, fmt=0)
    f.update(kw)
    return ac.q8_cache(**f)


def refused_by_all(ac, c, shape=SHAPE6):
    L = ac.lib()
    B, Hq, Hkv, d, ps, n = shape
    got = {L.ac_rope_kv_append_q8(P, P, P, P, c, P, 33, P, P, P, 513, *shape, None, None, None),
           L.ac_paged_decode_attn_q8(P, c, P, 33, P, 1, 0.0, 1, None, 0, P, *shape, 513, None, None, None),
           L.ac_kv_store_q8(P, P, c, P, 33, P, P, 5, B, Hkv, d, ps, n, None, None),
           L.ac_kv_load_q8(P, P, c, P, 33, P, P, 5, B, Hkv, d, ps, n, None, None)}
    assert len(got) == 1, got
    return got.pop()


@pytest.mark.parametrize("kw,want", [
    (dict(k_codes=None), NULL), (dict(v_codes=None), NULL), (dict(scales=None), NULL), (dict(fmt=2), UNSUPPORTED), (dict(fmt=-1), UNSUPPORTED),
    (dict(block=0), SHAPE), (dict(block=-16), SHAPE), (dict(block=8), UNSUPPORTED), (dict(block=24), UNSUPPORTED), (dict(block=64), SHAPE),
    (dict(stride_page=0), SHAPE), (dict(stride_token=-128), SHAPE), (dict(stride_token=120), ALIGN), (dict(stride_page=32 * 2 * 64 + 8), ALIGN),
    (dict(stride_token=48), SHAPE), (dict(stride_head=48), SHAPE), (dict(stride_page=1 << 40), UNSUPPORTED), (dict(stride_head=1 << 40), UNSUPPORTED),
    (dict(stride_scales=6), SHAPE), (dict(stride_scales=9), ALIGN), (dict(k_codes=P + 8), ALIGN), (dict(scales=P + 8), ALIGN)])
def test_descriptor_refusals(ac, kw, want):
    assert refused_by_all(ac, cache(ac, **kw)) == want


def test_shapes(ac):
    c = cache(ac)
    assert refused_by_all(ac, None) == NULL
    assert refused_by_all(ac, c, (1, 8, 2, 96, 32, 64)) == UNSUPPORTED and refused_by_all(ac, c, (0, 8, 2, 64, 32, 64)) == SHAPE
    assert refused_by_all(ac, c, (1, 8, 2, 64, 40, 64)) == UNSUPPORTED and refused_by_all(ac, c, (1, 8, 2, 64, 32, 0)) == SHAPE
    assert refused_by_all(ac, cache(ac, block=32, stride_scales=4), (1, 8, 2, 64, 48, 64)) == SHAPE


def test_call_refusals(ac):
    L, c = ac.lib(), cache(ac)
    assert L.ac_rope_kv_append_q8(None, P, P, P, c, P, 33, P, P, P, 513, *SHAPE6, None, None, None) == NULL
    assert L.ac_rope_kv_append_q8(P, P, P, P, c, P, 0, P, P, P, 513, *SHAPE6, None, None, None) == SHAPE
    assert L.ac_rope_kv_append_q8(P + 2, P, P, P, c, P, 33, P, P, P, 513, *SHAPE6, None, None, None) == ALIGN
    bad = ac._rope_options(rotary_dim=7)
    assert L.ac_rope_kv_append_q8(P, P, P, P, c, P, 33, P, P, P, 513, *SHAPE6, None, None, bad) == SHAPE

    def attn(q=P, splits=1, ws=None, wb=0, out=P, new=1, shape=SHAPE6, n=513, opt=None):
        return L.ac_paged_decode_attn_q8(q, c, P, 33, P, new, 0.0, splits, ws, wb, out, *shape, n, None, None, opt)

    assert attn(q=None) == NULL and attn(out=None) == NULL
    assert attn(n=0) == SHAPE and attn(splits=0) == SHAPE and attn(new=2) == UNSUPPORTED and attn(splits=65536) == UNSUPPORTED
    assert attn(shape=(1, 34, 2, 64, 32, 64)) == UNSUPPORTED and attn(shape=(1, 8, 3, 64, 32, 64)) == SHAPE
    assert attn(splits=4) == WORKSPACE and attn(splits=4, ws=P, wb=100) == WORKSPACE
    assert attn(splits=4, ws=P + 4, wb=1 << 20) == ALIGN and attn(q=P + 2) == ALIGN
    assert attn(opt=ac._options(window=-1)) == SHAPE and attn(opt=ac._options(window=4, sinks=-1)) == SHAPE
    assert attn(opt=ac._options(rope=ac._rope_options(rotary_dim=32))) == UNSUPPORTED
    assert L.ac_kv_store_q8(P, P, c, P, 33, P, P, -1, 1, 2, 64, 32, 64, None, None) == SHAPE
    assert L.ac_kv_store_q8(P, None, c, P, 33, P, P, 5, 1, 2, 64, 32, 64, None, None) == NULL
    assert L.ac_kv_load_q8(P, P + 8, c, P, 33, P, P, 5, 1, 2, 64, 32, 64, None, None) == ALIGN


@pytest.mark.parametrize("B,Hq,Hkv,n,lens", [(1, 8, 8, 100, None), (64, 32, 8, 8192, "ragged"), (4, 64, 8, 131072, None), (1, 8, 1, 2**31 - 1, None)])
def test_plans_cover_every_row(ac, B, Hq, Hkv, n, lens):
    counts = None if lens is None else [1 + (i * 7919) % n for i in range(B)]
    s, tokens, room = ac.ac_decode_plan_q8(counts, B, Hq, Hkv, 128, 16, n, 148)
    assert 1 <= s <= 65535 and tokens % 64 == 0 and s * tokens >= n and (s - 1) * tokens < n
    assert room == ac.ac_fused_workspace_bytes(B, Hq, Hkv, 128, s)
    out = [ctypes.c_int(), ctypes.c_int(), ctypes.c_size_t()]
    L = ac.lib()
    assert L.ac_decode_plan_q8(None, B, Hq, Hkv, 128, 16, 0, 148, *map(ctypes.byref, out)) == SHAPE
    assert L.ac_decode_plan_q8(None, B, Hq, Hkv, 128, 16, n, 148, None, ctypes.byref(out[1]), ctypes.byref(out[2])) == NULL
    with pytest.raises(ValueError):
        ac.ac_decode_plan_q8([1] * (B + 1), B, Hq, Hkv, 128, 16, n)


def test_table_refusals(ac):
    L, s = ac.lib(), ac.rope_scaling

    def tables(cos=P, sin=P, first=0, n=5, R=64, how=None):
        return L.ac_rope_tables(cos, sin, first, n, R, how if how is not None else s(), None)

    assert tables(cos=None) == NULL and tables(sin=None) == NULL and L.ac_rope_tables(P, P, 0, 5, 64, None, None) == NULL
    assert tables(n=-1) == SHAPE and tables(first=-1) == SHAPE and tables(R=0) == SHAPE and tables(R=7) == SHAPE
    assert tables(how=s(kind=4)) == UNSUPPORTED and tables(how=s(kind=-1)) == UNSUPPORTED
    nan = float("nan")
    for bad in (s(base=0.0), s(base=-1.0), s(base=nan), s(kind=1, factor=0.0), s(kind=1, factor=nan), s(kind=2, factor=-2.0), s(magnitude=-1.0), s(magnitude=nan),
                s(kind=3, factor=2.0, original=0.0, low=1.0, high=2.0), s(kind=3, factor=2.0, original=10.0, low=2.0, high=2.0),
                s(kind=3, factor=2.0, original=10.0, low=1.0, high=nan)):
        assert tables(how=bad) == SHAPE
    assert tables(R=2, how=s(kind=2, factor=2.0)) == SHAPE
    assert tables(cos=P + 4) == ALIGN


def test_row_refusals(ac):
    L = ac.lib()

    def rows(q=P, qo=2 * P, sq=512, sqo=512, k=3 * P, ko=4 * P, sk=128, sko=128, start=P, off=P, T=5, B=1, Hq=8, Hkv=2, d=64, cos=P, n=9, opt=None):
        return L.ac_rope_rows(q, qo, sq, sqo, k, ko, sk, sko, start, off, T, B, Hq, Hkv, d, cos, P, n, None, None, opt)

    for kw in (dict(q=None), dict(qo=None), dict(k=None), dict(ko=None), dict(start=None), dict(off=None), dict(cos=None)):
        assert rows(**kw) == NULL
    for kw in (dict(T=-1), dict(B=0), dict(Hq=0), dict(Hkv=-1), dict(d=0), dict(n=0), dict(sq=504), dict(sqo=511), dict(sk=120),
               dict(qo=P, sqo=520), dict(ko=3 * P, sko=136), dict(opt=ac._rope_options(rotary_dim=66)), dict(opt=ac._rope_options(rotary_dim=3))):
        assert rows(**kw) == SHAPE, kw
    for kw in (dict(sq=516), dict(sko=132), dict(q=P + 8), dict(ko=P + 2), dict(cos=P + 4)):
        assert rows(**kw) == ALIGN, kw
    for kw in (dict(d=96, sq=1024, sqo=1024, sk=512, sko=512), dict(B=65536), dict(Hq=65535, sq=1 << 23, sqo=1 << 23)):
        assert rows(**kw) == UNSUPPORTED, kw


def test_pools_that_are_copied_whole(ac):
    """Pages whose bytes do not follow the slots need not divide into them; the others still have to.  (A pool that is accepted
    meets the workspace, which is too small.)"""
    L = ac.lib()
    fork = lambda pool: L.ac_cache_fork(ac.page_pools([pool]), 1, P, 4, P, P, P, 1, 4, 32, 64, P, 0, None, None)      # noqa: E731
    assert fork((P, 16 * 17, 1)) == SHAPE and fork((P, 16 * 17, 1, 1)) == WORKSPACE and fork((P, 16 * 17, 1, 0)) == SHAPE
    assert fork((P, 256, 1)) == WORKSPACE and fork((P, 16, 1, 1)) == WORKSPACE
    assert fork((P, 8, 1, 1)) == ALIGN and fork((P, 0, 1, 1)) == SHAPE and fork((P + 8, 16, 1, 1)) == ALIGN
