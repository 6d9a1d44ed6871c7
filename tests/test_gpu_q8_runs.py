"""The 8-bit cache as a serving program uses it: prompts rotated and stored in pieces, forks, decode steps back to back and from
captured graphs, pages moved; several objects, streams and places far into a pool."""
import numpy as np
import pytest

from oracle import paged_decode_oracle as O
from oracle import q4_cache_oracle as A
from oracle import q8_cache_oracle as Q
from paper_2606_07665_b200 import workloads as W
from tests.test_gpu_q8 import Case, bits, check, dev, f64, host

pytestmark = pytest.mark.gpu

FORMATS = [Q.INT8, Q.E4M3]


@pytest.fixture(scope="module")
def rt():
    import torch
    from paper_2606_07665_b200 import build, runner
    build.build()
    torch.cuda.set_device(0)
    return runner


def kind(fmt):
    import torch
    return torch.int8 if fmt == Q.INT8 else torch.float8_e4m3fn


@pytest.mark.parametrize("fmt,Hkv,ps,block,layout", [(Q.E4M3, 2, 16, 16, "token_major"), (Q.INT8, 1, 48, 16, "head_major"), (Q.INT8, 3, 64, 32, "token_major")])
def test_a_conversation(rt, fmt, Hkv, ps, block, layout):
    """Two prompts, the first in two pieces; the second forked twice; all rows decode a few tokens; one is dropped, the pool compacted."""
    import torch
    d, Hq, rows, pages = 64, 4 * Hkv, 5, 40
    rng = np.random.default_rng(1)
    cache = rt.Q8Cache.empty(pages, ps, Hkv, d, block, kind(fmt), layout)
    rope = rt.Rope.scaled(512, d, base=10000.0, scaling="ramp", factor=8.0, original=64, low=1.0, high=4.0, magnitude=1.2)
    cos, sin = rope.cos.cpu().numpy(), rope.sin.cpu().numpy()
    table = torch.full((rows, 12), -1, dtype=torch.int32, device="cuda")
    lens = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
    refs = torch.zeros(pages, dtype=torch.int32, device="cuda")
    book = rt.CachePages(cache.pools, table, lens, refs, page_size=ps)
    lens[:2] = 0
    mirror = [[[], []] for _ in range(rows)]                       # what each row has been given, K (rotated) and V, bf16 bits
    want = Q.Cache(*(np.zeros((pages, ps, Hkv, d), np.uint8) for _ in range(2)), np.zeros((pages, Hkv, ps // block, 2), np.float32), fmt)

    def stored(row, x, start, t):
        for side in range(2):
            want.store(x[side], side, t, start)
            mirror[row][side].extend(x[side])

    for piece in ((30, 45), (23, 0)):                               # tokens of rows 0 and 1
        book.reserve(max(piece))
        q, k, v = (bits(rng, sum(piece), h, d) for h in (Hq, Hkv, Hkv))
        off = dev(np.array([0, piece[0], sum(piece)], np.int32))
        _, k_rot = rope.rows(dev(q), dev(k), lens[:2], off)
        cache.store(k_rot, dev(v), table[:2], lens[:2], off)
        torch.cuda.synchronize()
        t, n, at = table.cpu().numpy(), lens.cpu().numpy(), 0
        for b in range(2):
            xk = host(k_rot)[at:at + piece[b]]
            for i in range(piece[b]):
                for h in range(Hkv):
                    assert np.array_equal(xk[i, h], O.rope_rotate_variant_bf16(k[at + i, h], cos[n[b] + i], sin[n[b] + i], d, False))
            if piece[b]:
                stored(b, (xk, v[at:at + piece[b]]), int(n[b]), t[b])
            at += piece[b]
        lens[:2] += dev(np.array(piece, np.int32))
        book.trim()
    book.fork(dev(np.array([[1, 2], [1, 4]], np.int32)))
    torch.cuda.synchronize()
    assert int(book.status_flag) == 0
    t = table.cpu().numpy()
    for child in (2, 4):                                            # the oracle's copy of the partly filled page
        mirror[child] = [list(x) for x in mirror[1]]
        full, part = divmod(45, ps)
        if part:
            for side in range(2):
                want.pools[side][t[child, full], :part] = want.pools[side][t[1, full], :part]
            want.scales[t[child, full]] = want.scales[t[1, full]]
    step = rt.Q8DecodeStep(cache, table, lens, Hq, max_context_len=200, num_splits=2, rope_cos=rope.cos, rope_sin=rope.sin)
    q_in, k_new, v_new = (torch.zeros(rows, h, d, dtype=torch.int16, device="cuda") for h in (Hq, Hkv, Hkv))
    out, q_rot = torch.zeros(rows, Hq, d, dtype=torch.int16, device="cuda"), torch.zeros_like(q_in)
    step.step(q_in, k_new, v_new, q_rot, out)                       # outside the capture once: writes slots that the run writes again
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    book.reserve(1)
    with torch.cuda.graph(graph):
        step.step(q_in, k_new, v_new, q_rot, out)
    for i in range(2 * block + 3):
        if i:
            book.reserve(1)
        up = 2.0 ** rng.integers(-2, 3)
        q, k, v = bits(rng, rows, Hq, d), bits(rng, rows, Hkv, d, scale=up), bits(rng, rows, Hkv, d, scale=up)
        q_in.copy_(dev(q)), k_new.copy_(dev(k)), v_new.copy_(dev(v))
        graph.replay()
        torch.cuda.synchronize()
        t, n = table.cpu().numpy(), lens.cpu().numpy()
        for b in range(rows):
            if n[b] >= 0:
                kr = np.stack([O.rope_rotate_variant_bf16(k[b, h], cos[n[b]], sin[n[b]], d, False) for h in range(Hkv)])
                stored(b, (kr[None], v[b:b + 1]), int(n[b]), t[b])
        fetch = lambda b, h, pos: (lambda K, V: (K, V, np.abs(V)))(*(want.read(s, t[b], pos, h) for s in (0, 1)))      # noqa: E731
        ref, room = A.attention(host(q_rot), fetch, np.where(n >= 0, n + 1, 0), Hkv, slack=True)
        # products of up to 128 powers of two: 2^-11.6 of each weight, twice; the largest scale against a zero code as in Case.floor
        check(f64(out), ref, room * 3, i, 2.0**-31 * 200 * 448 * float(np.nanmax(want.scales)))
        lens[lens >= 0] += 1
        if i == block:
            book.release(dev(np.array([0], np.int32)))
            book.compact()
            torch.cuda.synchronize()
            t2 = table.cpu().numpy()
            moved = [(int(a), int(b)) for r in range(rows) if r != 0 and int(lens[r]) >= 0 for a, b in
                     zip(t[r, :-(-int(lens[r]) // ps)], t2[r, :-(-int(lens[r]) // ps)])]
            old = [p.copy() for p in want.pools], want.scales.copy()
            for a, b in moved:
                for side in range(2):
                    want.pools[side][b] = old[0][side][a]
                want.scales[b] = old[1][a]
    # what the rows hold is what they were given, within the format: a step of the final scale for codes rounded more than once
    for b in range(rows):
        n = int(lens[b])
        if n <= 0:
            continue
        t = table.cpu().numpy()
        for side in range(2):
            x = O.bf16_to_f64(np.array(mirror[b][side]))
            got = want.read(side, t[b], np.arange(n))
            pos = np.arange(n)
            s = want.scales[t[b, pos // ps], :, pos % ps // block, side].astype(np.float64)[..., None]
            err = np.abs(got - x)
            assert (err <= (s if fmt == Q.INT8 else np.maximum(2.0**-3 * np.abs(x), s * 2.0**-8))).all()
    assert int(book.status_flag) == 0 and int(step.status_flag) == 0 and int(cache.status_flag) == 0


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("splits", [1, 4])
def test_steps_back_to_back(rt, fmt, splits):
    """Each append may round codes again that the attention in front of it has read and the one behind it reads: the same bits as with a
    synchronisation after every call, with scales that grow at nearly every token."""
    import torch
    lens0 = [0, 3, 30, 500, 1000, 65]
    c = Case(3, lens0, 8, 2, 128, 32, 32, fmt, room=40)
    cos, sin = W.rope_table(1100, 128, 10000.0)
    q, k, v = (dev(bits(np.random.default_rng(5), 36, 6, h, 128)).view(torch.bfloat16) for h in (8, 2, 2))
    k, v = (x * torch.pow(1.3, torch.arange(36, device="cuda") - 18.0)[:, None, None, None].bfloat16() for x in (k, v))
    results = []
    for wait in (True, False):
        cache, lens = c.upload(rt), dev(c.lens)
        step = rt.Q8DecodeStep(cache, dev(c.table), lens, 8, max_context_len=1050, num_splits=splits, rope_cos=dev(cos), rope_sin=dev(sin))
        out = torch.zeros(36, 6, 8, 128, device="cuda").bfloat16()
        torch.cuda.synchronize()
        for i in range(36):
            q_rot = step.append(q[i], k[i], v[i])
            if wait:
                torch.cuda.synchronize()
            step.attention(q_rot, out=out[i])
            if wait:
                torch.cuda.synchronize()
            lens += 1
        torch.cuda.synchronize()
        results.append((out, cache.k_codes, cache.v_codes, cache.scales))
    for a, b in zip(*results):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_objects_on_streams_of_their_own(rt):
    """Two steps over one cache, each with its workspace and stream, and outputs that are allocated for the stream."""
    import torch
    c = Case(4, [700, 900], 8, 2, 64, 16, 16, Q.INT8)
    cache = c.upload(rt)
    q = dev(bits(c.rng, 2, 8, 64))
    steps = [rt.Q8DecodeStep(cache, dev(c.table), dev(c.lens), 8, lens_host=c.lens, num_splits=n) for n in (3, 5)]
    alone = [s.attention(q) for s in steps]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in steps]
    got = [[s.attention(q, stream=t if i % 2 else t.cuda_stream) for s, t in zip(steps, streams)] for i in range(20)]
    torch.cuda.synchronize()
    for pair in got:
        for a, b in zip(pair, alone):
            assert torch.equal(a, b)


def test_plans_of_captured_calls_stay(rt):
    import torch
    c = Case(5, [700, 900], 8, 2, 64, 16, 16, Q.E4M3)
    q = dev(bits(c.rng, 2, 8, 64))
    step = rt.Q8DecodeStep(c.upload(rt), dev(c.table), dev(c.lens), 8, lens_host=c.lens, num_splits=4)
    want = step.attention(q).clone()
    out = torch.zeros_like(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step.attention(q, out=out)
    step.plan(c.lens, num_splits=2)
    step.attention(q)
    junk = [torch.full((1 << 18,), 7.0, device="cuda") for _ in range(8)]      # whatever memory the first plan gave up
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want) and len(junk) == 8


@pytest.mark.parametrize("fmt", FORMATS)
def test_pages_past_4_gb(rt, fmt):
    """The same rows in the first pages of a pool and in those behind 2^32 bytes of codes: the same bits from every call."""
    import torch
    Hkv, d, ps, Hq = 8, 128, 64, 16
    need = (1 << 32) // (ps * Hkv * d) + 70
    c = Case(6, [200, 1500, 63], Hq, Hkv, d, ps, 16, fmt, room=2)
    big = rt.Q8Cache.empty(need, ps, Hkv, d, 16, kind(fmt))
    small = c.upload(rt)
    shift = need - c.num_pages
    for a, b in ((big.k_codes, small.k_codes), (big.v_codes, small.v_codes)):
        a.view(torch.uint8)[shift:].copy_(b.view(torch.uint8))
    big.scales[shift:].copy_(small.scales)
    cos, sin = W.rope_table(1600, d, 10000.0)
    rng = np.random.default_rng(8)
    q, k, v = (dev(bits(rng, 3, h, d)) for h in (Hq, Hkv, Hkv))
    xs = [dev(bits(rng, 30, Hkv, d)) for _ in range(2)]
    off = dev(np.array([0, 10, 20, 30], np.int32))
    results = []
    for cache, table in ((small, c.table), (big, np.where(c.table >= 0, c.table + shift, c.table))):
        table = dev(table)
        step = rt.Q8DecodeStep(cache, table, dev(c.lens), Hq, lens_host=c.lens, rope_cos=dev(cos), rope_sin=dev(sin))
        outs = [step.step(q, k, v)]
        cache.store(*xs, table, dev(c.lens - 20), off)
        outs += cache.load(table, dev(c.lens - 30), off, 30)
        results.append(outs + [t.view(torch.uint8)[-c.num_pages:] for t in (cache.k_codes, cache.v_codes)])
        assert int(cache.status_flag) == 0 and int(step.status_flag) == 0
    for a, b in zip(*results):
        assert torch.equal(a, b)


def test_strides_of_the_callers(rt):
    """Codes and scales inside larger tensors, pages and tokens further apart than they are long."""
    import ctypes

    import torch
    from paper_2606_07665_b200 import binding as ac
    c = Case(9, [100, 37], 4, 2, 64, 32, 16, Q.INT8, room=3)
    pad = torch.full((2, c.num_pages, 32 + 3, 2 + 1, 64 + 16), 0x55, dtype=torch.uint8, device="cuda")
    sc = torch.full((c.num_pages, 2 * 2 * 2 + 6), 5.0, device="cuda")
    for side in range(2):
        pad[side, :, :32, :2, :64] = dev(c.cache.pools[side])
    sc[:, :8] = dev(c.cache.scales).reshape(c.num_pages, 8)
    s = ac.q8_cache(pad[0], pad[1], sc, pad.stride(1), pad.stride(2), pad.stride(3), sc.stride(0), 16, ac.AC_Q8_INT8)
    q, k, v = (dev(bits(c.rng, 2, h, 64)) for h in (4, 2, 2))
    cos, sin = W.rope_table(200, 64, 10000.0)
    table, lens = dev(c.table), dev(c.lens)
    shape = (2, 4, 2, 64, 32, c.num_pages)
    q_rot, out = torch.zeros_like(q), torch.zeros_like(q)
    ac.ac_rope_kv_append_q8(q, q_rot, k, v, s, table, c.table.shape[1], lens, dev(cos), dev(sin), 200, *shape)
    ac.ac_paged_decode_attn_q8(q_rot, s, table, c.table.shape[1], lens, 1, 0.0, 1, None, 0, out, *shape, 101)
    off, start = dev(np.array([0, 1, 2], np.int32)), dev(c.lens + 1)
    ac.ac_kv_store_q8(v, k, s, table, c.table.shape[1], start, off, 2, 2, 2, 64, 32, c.num_pages)
    kb, vb = torch.zeros_like(k), torch.zeros_like(v)
    ac.ac_kv_load_q8(kb, vb, s, table, c.table.shape[1], start, off, 2, 2, 2, 64, 32, c.num_pages)
    dense = c.upload(rt)
    step = rt.Q8DecodeStep(dense, table, lens, 4, lens_host=c.lens, num_splits=1, rope_cos=dev(cos), rope_sin=dev(sin))
    assert torch.equal(step.step(q, k, v), out)
    dense.store(v, k, table, start, off)
    assert all(torch.equal(a.view(torch.int16), b) for a, b in zip(dense.load(table, start, off, 2), (kb, vb)))
    for side, pool in enumerate((dense.k_codes, dense.v_codes)):
        assert torch.equal(pad[side, :, :32, :2, :64], pool.view(torch.uint8))
    assert (pad[:, :, 32:] == 0x55).all() and (pad[:, :, :, 2:] == 0x55).all() and (pad[..., 64:] == 0x55).all() and (sc[:, 8:] == 5).all()
    assert ctypes.sizeof(s) == 72


def test_object_refusals(rt):
    import torch
    e = rt.Q8Cache.empty(4, 32, 2, 64, 16, torch.int8)
    k, v, s = e.k_codes, e.v_codes, e.scales
    for bad in ((k.view(torch.uint8), v, s), (k, v.view(torch.float8_e4m3fn), s), (k, v[:, :16], s), (k, v, s.double()), (k, v, s[:, :1]),
                (k, v, s[:3]), (k[0], v, s), (k, v, s[0]), (k, v, s.transpose(1, 2)), (k, v, torch.zeros(4, 2, 5, 2, device="cuda"))):
        with pytest.raises(ValueError):
            rt.Q8Cache(*bad)
    with pytest.raises(ValueError):
        rt.Q8Cache(k, v, s, layout="slot_major")
    with pytest.raises(ValueError):
        rt.Q8Cache(k, v, s, page_size=16)
    for kw in (dict(block=8), dict(block=24), dict(block=0), dict(dtype=torch.uint8)):
        with pytest.raises(ValueError):
            rt.Q8Cache.empty(4, 32, 2, 64, **kw)
    table, lens = torch.zeros(1, 4, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    with pytest.raises(TypeError):
        rt.Q4DecodeStep(e, table, lens, 4)
    with pytest.raises(TypeError):
        rt.Q8DecodeStep(rt.Q4Cache.empty(4, 32, 2, 64), table, lens, 4)
    step = rt.Q8DecodeStep(e, table, lens, 4)
    with pytest.raises(ValueError):
        step.append(*[torch.zeros(1, h, 64, dtype=torch.bfloat16, device="cuda") for h in (4, 2, 2)])
    with pytest.raises(ValueError):
        step.attention(torch.zeros(1, 4, 64, device="cuda"))
    odd = rt.Q8Cache(torch.zeros(3, 16, 1, 64, dtype=torch.int8, device="cuda"), torch.zeros(3, 16, 1, 64, dtype=torch.int8, device="cuda"),
                     torch.zeros(3, 1, 1, 2, device="cuda"))
    with pytest.raises(ValueError):
        odd.pools
    assert [tuple(p[0].shape) for p in rt.Q8Cache.empty(3, 16, 1, 64).pools][2] == (3, 4)


def test_rope_refusals(rt):
    import torch
    f = lambda *s: torch.zeros(*s, device="cuda")                                                 # noqa: E731
    b = lambda *s: torch.zeros(*s, device="cuda", dtype=torch.bfloat16)                           # noqa: E731
    i = lambda *s: torch.zeros(*s, device="cuda", dtype=torch.int32)                              # noqa: E731
    for bad in (dict(cos=f(8, 32), sin=f(8, 31)), dict(cos=f(8), sin=f(8)), dict(cos=f(8, 32).double(), sin=f(8, 32).double()),
                dict(cos=f(8, 32), sin=f(8, 32), rotary_dim=32), dict(cos=f(8, 64)[:, ::2], sin=f(8, 64)[:, ::2])):
        with pytest.raises(ValueError):
            rt.Rope(**bad)
    for kw in (dict(max_position=0), dict(rotary_dim=7), dict(scaling="cubic")):
        with pytest.raises(ValueError):
            rt.Rope.scaled(**{**dict(max_position=8, rotary_dim=64), **kw})
    from paper_2606_07665_b200 import binding as ac
    for kw in (dict(base=0.0), dict(scaling="linear", factor=0.0), dict(scaling="ramp", factor=2.0), dict(magnitude=-1.0), dict(first_position=-1)):
        with pytest.raises(ac.AcError):
            rt.Rope(f(8, 32), f(8, 32)).fill(**kw)
    r = rt.Rope(f(8, 32), f(8, 32))
    q, k, start, off = b(5, 4, 64), b(5, 2, 64), i(1), i(2)
    assert [t.shape for t in r.rows(q, k, start, off)] == [q.shape, k.shape]
    for bad in ((q.float(), k, start, off), (q[:4], k, start, off), (q, k[:, :, :32], start, off), (q, k, start.long(), off), (q, k, start, i(3)),
                (b(5, 64, 4).transpose(1, 2), k, start, off), (q[0], k, start, off)):
        with pytest.raises(ValueError):
            r.rows(*bad)
    with pytest.raises(ValueError):
        r.rows(q, k, start, off, q_out=b(5, 4, 128))
    with pytest.raises(ac.AcError):                                                               # heads of 32 are not supported
        r.rows(b(5, 4, 32), None, start, off)
    with pytest.raises(ValueError):
        rt.Rope(f(8, 32), f(8, 32), q_norm_weight=b(128)).rows(q, k, start, off)
    q0, k0 = r.rows(b(0, 4, 64), b(0, 2, 64), start, off)
    assert q0.shape == (0, 4, 64) and k0.shape == (0, 2, 64)


def test_rope_refuses_what_is_no_tensor(rt):
    import torch
    r = rt.Rope(torch.zeros(8, 32, device="cuda"), torch.zeros(8, 32, device="cuda"))
    q = torch.zeros(5, 4, 64, device="cuda", dtype=torch.bfloat16)
    start, off = torch.zeros(1, device="cuda", dtype=torch.int32), torch.zeros(2, device="cuda", dtype=torch.int32)
    for bad in ((q, None, None, off), (q, None, start, [0, 5]), (q, [q], start, off), (q, None, 0, off)):
        with pytest.raises(TypeError):
            r.rows(*bad)
    with pytest.raises(ValueError):
        r.rows(q, None, start[0], off)
    with pytest.raises(ValueError):
        r.rows(q, None, start, off[0])
