"""Host-side checks, no GPU: the plans and refusals of the 4-bit cache, the sinks and the page operations, and the pins
of their oracle."""
import ctypes

import numpy as np
import pytest

from oracle import paged_decode_oracle as O
from oracle import q4_cache_oracle as Q

P = 0x10000            # fake, aligned, never dereferenced: every call below is refused before a launch
NULL, SHAPE, UNSUPPORTED, ALIGN, WORKSPACE = 1, 2, 3, 4, 5


@pytest.fixture(scope="module")
def ac():
    from paper_2606_07665_b200 import binding, build
    build.build()
    binding.lib()
    return binding


def cache(ac, **kw):
    c = dict(k_codes=P, v_codes=P, params=P, stride_page=1024, stride_token=64, stride_head=32, group=64)
    c.update(kw)
    return ac.AcQ4Cache(*[c[k] for k in ("k_codes", "v_codes", "params", "stride_page", "stride_token", "stride_head", "group")])


def test_window_span(ac):
    assert ac.ac_window_span(0, 5) == 2**31 - 1 and ac.ac_window_span(-3) == 2**31 - 1
    assert ac.ac_window_span(100) == 163
    assert ac.ac_window_span(100, 1) == 179 and ac.ac_window_span(100, 16) == 179 and ac.ac_window_span(100, 17) == 195
    assert ac.ac_window_span(2**31 - 1, 2**31 - 1) == 2**31 - 1


@pytest.mark.parametrize("B,Hq,Hkv,d,ps,n", [(1, 8, 2, 64, 16, 1), (1, 32, 8, 128, 16, 4097), (64, 32, 8, 128, 16, 8192),
                                             (4, 64, 8, 128, 16, 131073), (256, 28, 4, 128, 32, 2049), (1, 8, 1, 64, 16, 2**30)])
def test_plan_q4(ac, B, Hq, Hkv, d, ps, n):
    for counts in (None, [n] * B, [1] * B, [0] * B, [n] + [-1] * (B - 1)):
        S, st, wb = ac.ac_decode_plan_q4(counts, B, Hq, Hkv, d, ps, n, 148)
        assert S >= 1 and st % 64 == 0 and st * S >= n and st * (S - 1) < n
        assert wb == ac.ac_fused_workspace_bytes(B, Hq, Hkv, d, S)
    L = ac.lib()
    ns, sp, w = ctypes.c_int(), ctypes.c_int(), ctypes.c_size_t()
    a = (ctypes.byref(ns), ctypes.byref(sp), ctypes.byref(w))
    assert L.ac_decode_plan_q4(None, 1, 8, 2, 64, 16, 512, 148, None, None, None) == NULL
    assert L.ac_decode_plan_q4(None, 0, 8, 2, 64, 16, 512, 148, *a) == SHAPE
    assert L.ac_decode_plan_q4(None, 1, 8, 2, 96, 16, 512, 148, *a) == UNSUPPORTED
    assert L.ac_decode_plan_q4(None, 1, 8, 2, 64, 16, 0, 148, *a) == SHAPE
    with pytest.raises(ValueError):
        ac.ac_decode_plan_q4([5, 6], 3, 8, 2, 64, 16, 512)


SHAPE6 = (1, 8, 2, 64, 16, 64)


@pytest.mark.parametrize("kw,want", [
    (dict(k_codes=None), NULL), (dict(params=None), NULL), (dict(group=48), UNSUPPORTED), (dict(group=128), UNSUPPORTED),
    (dict(group=0), UNSUPPORTED), (dict(stride_token=40), ALIGN), (dict(stride_token=16), SHAPE), (dict(stride_head=16), SHAPE),
    (dict(stride_page=-16), SHAPE), (dict(v_codes=P + 8), ALIGN), (dict(params=P + 4), ALIGN)])
def test_q4_cache_descriptor_refusals(ac, kw, want):
    L, c = ac.lib(), cache(ac, **kw)
    assert L.ac_rope_kv_append_q4(P, P, P, P, c, P, 33, P, P, P, 513, *SHAPE6, None, None, None) == want
    assert L.ac_paged_decode_attn_q4(P, c, P, 33, P, 1, 0.0, 1, None, 0, P, *SHAPE6, 513, None, None, None) == want
    assert L.ac_kv_store_q4(P, P, c, P, 33, P, P, 5, 1, 2, 64, 16, 64, None, None) == want
    assert L.ac_kv_load_q4(P, P, c, P, 33, P, P, 5, 1, 2, 64, 16, 64, None, None) == want


def test_q4_call_refusals(ac):
    L, c = ac.lib(), cache(ac)
    assert L.ac_rope_kv_append_q4(None, P, P, P, c, P, 33, P, P, P, 513, *SHAPE6, None, None, None) == NULL
    assert L.ac_rope_kv_append_q4(P, P, P, P, None, P, 33, P, P, P, 513, *SHAPE6, None, None, None) == NULL
    assert L.ac_rope_kv_append_q4(P, P, P, P, c, P, 0, P, P, P, 513, *SHAPE6, None, None, None) == SHAPE
    assert L.ac_rope_kv_append_q4(P + 2, P, P, P, c, P, 33, P, P, P, 513, *SHAPE6, None, None, None) == ALIGN
    assert L.ac_rope_kv_append_q4(P, P, P, P, c, P, 33, P, P, P, 513, 1, 8, 2, 64, 24, 64, None, None, None) == UNSUPPORTED
    bad = ac._rope_options(rotary_dim=7)
    assert L.ac_rope_kv_append_q4(P, P, P, P, c, P, 33, P, P, P, 513, *SHAPE6, None, None, bad) == SHAPE

    def attn(q=P, splits=1, ws=None, wb=0, out=P, new=1, shape=SHAPE6, n=513, opt=None):
        return L.ac_paged_decode_attn_q4(q, c, P, 33, P, new, 0.0, splits, ws, wb, out, *shape, n, None, None, opt)

    assert attn(q=None) == NULL and attn(out=None) == NULL
    assert attn(n=0) == SHAPE and attn(splits=0) == SHAPE and attn(new=2) == UNSUPPORTED
    assert attn(shape=(1, 34, 2, 64, 16, 64)) == UNSUPPORTED and attn(shape=(1, 8, 3, 64, 16, 64)) == SHAPE
    assert attn(splits=4) == WORKSPACE and attn(splits=4, ws=P, wb=100) == WORKSPACE
    assert attn(splits=4, ws=P + 4, wb=1 << 20) == ALIGN and attn(q=P + 2) == ALIGN
    far = cache(ac, stride_page=1 << 31)                                        # 64 pages of 2 GB: more than 2^36 bytes
    assert L.ac_paged_decode_attn_q4(P, far, P, 33, P, 1, 0.0, 1, None, 0, P, *SHAPE6, 513, None, None, None) == UNSUPPORTED
    assert attn(opt=ac._options(window=-1)) == SHAPE and attn(opt=ac._options(window=4, sinks=-1)) == SHAPE
    assert attn(opt=ac._options(rope=ac._rope_options(rotary_dim=32))) == UNSUPPORTED
    assert L.ac_kv_store_q4(P, P, c, P, 33, P, P, -1, 1, 2, 64, 16, 64, None, None) == SHAPE
    assert L.ac_kv_store_q4(P, None, c, P, 33, P, P, 5, 1, 2, 64, 16, 64, None, None) == NULL
    assert L.ac_kv_load_q4(P, P + 8, c, P, 33, P, P, 5, 1, 2, 64, 16, 64, None, None) == ALIGN
    assert L.ac_kv_load_q4(P, P, c, P, 33, P, P, 5, 0, 2, 64, 16, 64, None, None) == SHAPE


def test_sinks_refusals_of_the_bf16_entry_points(ac):
    L = ac.lib()
    o = ac._options(window=8, sinks=-1)
    assert L.ac_paged_decode_attn_ex(P, P, P, 2048, 128, 64, P, 33, P, 1, 0.0, 1, None, 0, P, *SHAPE6, 513, None, None, o) == SHAPE
    assert L.ac_decode_step_fused_ex(P, None, P, P, P, P, 2048, 128, 64, P, 33, P, P, P, 513, 0.0, 1, None, 0, P, *SHAPE6, 513,
                                     None, None, o) == SHAPE


def test_page_call_refusals(ac):
    L = ac.lib()
    pools = lambda *p: ac.page_pools(list(p))                                  # noqa: E731
    good = pools((P, 4096, 1))
    wb = ac.ac_cache_workspace_bytes(4, 64, 4)
    assert wb >= 64 * 8 and ac.ac_cache_workspace_bytes(0, 64, 4) == 0
    assert L.ac_cache_copy_pages(good, 1, None, 1, 64, None, None) == NULL
    assert L.ac_cache_copy_pages(None, 1, P, 1, 64, None, None) == NULL
    assert L.ac_cache_copy_pages(good, 0, P, 1, 64, None, None) == SHAPE
    assert L.ac_cache_copy_pages(good, 129, P, 1, 64, None, None) == UNSUPPORTED
    assert L.ac_cache_copy_pages(good, 1, P, -1, 64, None, None) == SHAPE
    assert L.ac_cache_copy_pages(good, 1, P + 4, 1, 64, None, None) == ALIGN
    for bad, want in (((P, 0, 1), SHAPE), ((P, 4096, 0), SHAPE), ((P + 8, 4096, 1), ALIGN), ((P, 4096 + 8, 1), ALIGN),
                      ((P, 48, 2), ALIGN), ((None, 4096, 1), NULL)):
        assert L.ac_cache_copy_pages(pools(bad), 1, P, 1, 64, None, None) == want

    def reserve(table=P, mp=8, new=1, rows=4, ps=16, pages=64, ws=P, n=wb, refs=P):
        return L.ac_cache_reserve(table, mp, P, refs, new, rows, ps, pages, ws, n, None, None)

    assert reserve(table=None) == NULL and reserve(mp=0) == SHAPE and reserve(new=-1) == SHAPE and reserve(rows=0) == SHAPE
    assert reserve(ps=0) == SHAPE and reserve(pages=2**30 + 1) == UNSUPPORTED and reserve(ws=None) == WORKSPACE
    assert reserve(n=100) == WORKSPACE and reserve(refs=P + 4) == ALIGN

    def fork(pl=good, np_=1, n=4, ws=P, size=wb, pairs=P, ps=16):
        return L.ac_cache_fork(pl, np_, P, 8, P, P, pairs, n, 4, ps, 64, ws, size, None, None)

    assert fork(pairs=None) == NULL and fork(n=-1) == SHAPE and fork(ws=None) == WORKSPACE and fork(size=64) == WORKSPACE
    assert fork(ps=48) == SHAPE                                                 # 4096 bytes are not 48 equal slots
    assert fork(pairs=P + 4) == ALIGN
    assert L.ac_cache_release(P, 8, P, P, None, 1, 4, 16, 64, None, None) == NULL
    assert L.ac_cache_release(P, 8, P, P, P, -1, 4, 16, 64, None, None) == SHAPE
    assert L.ac_cache_compact(good, 1, P, P + 64, 8, P, P, P, 4, 16, 64, None, P, wb, None, None) == UNSUPPORTED
    assert L.ac_cache_compact(good, 1, P, P, 8, P, P, P, 4, 16, 64, None, P, 10, None, None) == WORKSPACE
    assert L.ac_cache_compact(good, 1, None, P, 8, P, P, P, 4, 16, 64, None, P, wb, None, None) == NULL


def test_runner_refuses_tensors_off_the_gpu():
    import torch
    from paper_2606_07665_b200 import runner
    codes, params = torch.zeros(4, 16, 2, 32, dtype=torch.uint8), torch.zeros(4, 2, 16, 2, 1, 2, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="CUDA"):
        runner.Q4Cache(codes, codes, params)
    with pytest.raises(ValueError, match="CUDA"):
        runner.CachePages([codes], torch.zeros(2, 4, dtype=torch.int32), torch.zeros(2, dtype=torch.int32),
                          torch.zeros(4, dtype=torch.int32), 16)
    kv = torch.zeros(4, 16, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="CUDA"):
        runner.PagedAttention(kv, kv, torch.zeros(2, 4, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), 8)


# ---- pins of the oracle -----------------------------------------------------------------------------------------


def test_oracle_quantiser_pins():
    # sixteen equidistant values are their own codes; the steps are exact
    x = O.f64_to_bf16_rne(np.arange(32) % 16 * 0.25 - 1.0)
    c, s, m = Q.quantise(x, 32)
    assert (c == np.arange(32) % 16).all() and O.bf16_to_f64(s) == 0.25 and O.bf16_to_f64(m) == -1.0
    assert (Q.values(Q.pack(c), s, m)[0] == O.bf16_to_f64(x)).all()
    assert (Q.unpack(Q.pack(c)) == c).all()
    # ties go to the even code: 0.5 and 1.5 steps
    y = np.zeros(32)
    y[:4] = [15.0, 0.5, 1.5, 2.5]
    c, s, m = Q.quantise(O.f64_to_bf16_rne(y), 32)
    assert O.bf16_to_f64(s) == 1.0 and list(c[:4]) == [15, 0, 2, 2]
    # a constant group, a group with a NaN
    c, s, m = Q.quantise(np.array([0x3F80] * 32 + [0x7F80] + [0x3F80] * 31, dtype=np.uint16), 32)
    assert list(s) == [0, 0] and list(m) == [0x3F80, 0x7FC0] and not c.any()
    # half a step at most, plus the scale's own rounding
    g = np.random.default_rng(0)
    x = O.f64_to_bf16_rne(g.standard_normal((50, 128)))
    c, s, m = Q.quantise(x, 64)
    err = np.abs(Q.values(Q.pack(c), s, m)[0] - O.bf16_to_f64(x))
    assert (err <= np.repeat(O.bf16_to_f64(s), 64, -1) * (0.5 + 15 * 2.0**-8)).all()


def test_oracle_visible_and_attention_agree_with_the_bf16_oracle():
    from paper_2606_07665_b200 import workloads as W
    assert list(Q.visible(6, 2, 1)) == [0, 4, 5] and list(Q.visible(3, 5, 1)) == [0, 1, 2] and list(Q.visible(0, 2, 1)) == []
    w = W.make_workload("t", 3, B=2, Hq=4, Hkv=2, d=64, page_size=16, num_pages=20, context_lens=[40, 7], rope_base=1e4)

    def fetch(b, h, t):
        pg, sl = w.block_table[b, t // 16], t % 16
        return O.bf16_to_f64(w.k_cache[pg, sl, h]), O.bf16_to_f64(w.v_cache[pg, sl, h]), np.zeros((len(t), 64))

    for window in (0, 5, 33):
        ref = O.oracle_paged_decode_attn(w.q, w.k_cache, w.v_cache, w.block_table, w.context_lens, 16, new_tokens=0, window=window)
        assert np.allclose(Q.attention(w.q, fetch, w.context_lens, 2, window), ref, atol=1e-12)


def test_oracle_pages_invariants():
    g = np.random.default_rng(1)
    lens = np.array([40, 16, 0, 33, -1, -1], dtype=np.int32)
    table = np.full((6, 5), 63, dtype=np.int32)
    refs = np.zeros(64, dtype=np.int32)
    perm = g.permutation(63)
    at = 0
    for r, n in enumerate(lens):
        k = -(-max(n, 0) // 16)
        table[r, :k] = perm[at:at + k]
        refs[perm[at:at + k]] = 1
        at += k
    pool = g.integers(0, 255, (64, 16, 4))
    o = Q.Pages(table, lens, refs, 16, [(pool, 1)])
    read = lambda r: np.concatenate([o.pools[0][0][o.table[r, i // 16], i % 16] for i in range(max(o.lens[r], 0))] or [np.zeros(0)])  # noqa: E731
    before = [read(r) for r in range(4)]
    o.fork([(0, 4), (3, 5)])
    assert (read(4) == before[0]).all() and (read(5) == before[3]).all() and o.table[4, 2] != o.table[0, 2]
    assert o.refs.sum() == 3 + 1 + 3 + 3 + 3 and o.refs[o.table[0, 0]] == 2
    o.reserve(30)
    o.release([0, 0])
    live = o.compact()
    assert (o.refs[:live] > 0).all() and not o.refs[live:].any()
    assert (read(4) == before[0]).all() and (read(1) == before[1]).all() and (read(5) == before[3]).all()
