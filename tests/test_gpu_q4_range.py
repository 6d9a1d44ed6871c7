"""4-bit attention at the ends of its stated range."""
import numpy as np
import pytest

from paper_2606_07665_b200 import workloads as W
from tests.test_gpu_q4 import Case, run_attention

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rt():
    import torch
    from paper_2606_07665_b200 import build, runner
    build.build()
    torch.cuda.set_device(0)
    return runner


@pytest.mark.parametrize("splits", [1, 3])
@pytest.mark.parametrize("Hq", [8, 24])
def test_values_as_large_as_the_sums_allow(rt, Hq, splits):
    """800 tokens of |V| below 2^108 are 2^118, the stated limit; scores that creep up by less than the reference's lag keep
    the weights as large as they get."""
    c = Case(rt, 130, [799], Hq, 2, 128, 16, 64, v_scale=2.0**105)
    q = W.f32_to_bf16_bits(np.abs(c.rng.standard_normal((1, Hq, 128))).astype(np.float32))
    for t in range(800):
        c.prm[c.table[0, t // 16], :, t % 16, 0, :, 1] = W.f32_to_bf16_bits(np.full((2, 2), -7.5 * 0.2 + 0.05 * t / 800, np.float32))
    top = max(np.abs(c.fetch(0, h, np.arange(800))[1]).max() for h in range(2))
    assert 2.0**106 < top and 800 * top < 2.0**118
    run_attention(rt, c, q=q, splits=splits)


@pytest.mark.parametrize("layout", ["pages far apart", "slots far apart"])
def test_places_past_32_bits(rt, layout):
    """Code pools of 36 GB (one allocation, of which little is touched): places beyond 2^32 bytes, and beyond 2^31 units
    of 16 bytes, are written, read back and attended."""
    import torch
    from oracle import q4_cache_oracle as Q
    from paper_2606_07665_b200 import binding as ac
    from tests.test_gpu_q4 import bits, check, dev, f64
    rng = np.random.default_rng(131)
    B, Hq, Hkv, d, group, ps, num_pages = 2, 8, 2, 128, 64, 32, 70
    total = 36 << 30
    if layout == "pages far apart":
        page, token, head = 1 << 29, Hkv * d // 2, d // 2
    else:                                                  # [slot, page, head, byte], a slot's pages a gigabyte from the next's
        page, token, head = Hkv * d // 2, 1 << 30, d // 2
    side = 1 << 20                                         # V's pool lies a megabyte behind K's, in the same allocation
    assert (num_pages - 1) * page + (ps - 1) * token + side + Hkv * d <= total and (num_pages - 1) * page + 16 * token > 1 << 33
    memory = torch.empty(total, dtype=torch.uint8, device="cuda")
    params = torch.zeros(num_pages, Hkv, ps, 2, d // group, 2, dtype=torch.bfloat16, device="cuda")
    c = ac.q4_cache(memory.data_ptr(), memory.data_ptr() + side, params, page, token, head, group)
    table = dev(np.array([[69, 2, 66], [67, 0, 68]], dtype=np.int32))
    lens = np.array([90, 70], dtype=np.int32)
    off, zero = dev(np.array([0, 90, 160], dtype=np.int32)), dev(np.zeros(B, np.int32))
    k, v = bits(rng, 160, Hkv, d), bits(rng, 160, Hkv, d)
    flag = dev(np.zeros(1, np.int32))
    ac.ac_kv_store_q4(dev(k), dev(v), c, table, 3, zero, off, 160, B, Hkv, d, ps, num_pages, flag)
    kb, vb = (torch.zeros(160, Hkv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ac.ac_kv_load_q4(kb, vb, c, table, 3, zero, off, 160, B, Hkv, d, ps, num_pages, flag)
    cos, sin = torch.ones(128, d // 2, device="cuda"), torch.zeros(128, d // 2, device="cuda")     # no rotation
    q, kn, vn = bits(rng, B, Hq, d), bits(rng, B, Hkv, d), bits(rng, B, Hkv, d)
    q_rot, out = dev(q).clone(), dev(q).clone()
    ac.ac_rope_kv_append_q4(dev(q), q_rot, dev(kn), dev(vn), c, table, 3, dev(lens), cos, sin, 128, B, Hq, Hkv, d, ps, num_pages, flag)
    ac.ac_paged_decode_attn_q4(q_rot, c, table, 3, dev(lens), 1, 0.0, 1, None, 0, out, B, Hq, Hkv, d, ps, num_pages, 96, flag)
    torch.cuda.synchronize()
    assert int(flag) == 0
    held = []
    for x, new, back in ((k, kn, kb), (v, vn, vb)):
        codes, s, m = Q.quantise(np.concatenate([x, new]), group)
        held.append(Q.values(Q.pack(codes), s, m))
        want = held[-1][0][:160]
        assert (np.abs(back.double().cpu().numpy() - want) <= 2.0**-8 * (1 + 2.0**-8) * np.abs(want)).all()

    def fetch(b, h, t):
        at = np.where(t < lens[b], [0, 90][b] + t, 160 + b)
        (K, _), (V, cs) = held
        return K[at, h], V[at, h], np.abs(cs[at, h]) + np.abs(V[at, h]) / 8

    ref, room = Q.attention(q, fetch, lens + 1, Hkv, slack=True)
    check(f64(out), ref, room, layout)
    del memory, c
    torch.cuda.empty_cache()


def test_page_copies_past_32_bits(rt):
    import torch
    num_pages, page = 9000, 1 << 20                        # 9.4 GB, of which a few pages are looked at
    pool = torch.empty(num_pages, 16, page // 16, dtype=torch.uint8, device="cuda")
    marks = {8999: 1, 4096: 2, 8191: 3, 5: 4}
    for p, x in marks.items():
        pool[p] = x
    lens = torch.tensor([2 * 16 + 8, 16, -1], dtype=torch.int32, device="cuda")
    table = torch.tensor([[8999, 4096, 8191, 0], [5, 0, 0, 0], [0, 0, 0, 0]], dtype=torch.int32, device="cuda")
    refs = torch.zeros(num_pages, dtype=torch.int32, device="cuda")
    refs[list(marks)] = 1
    h = rt.CachePages([pool], table, lens, refs, 16)
    h.copy(torch.tensor([[8999, 7000], [5, 8998]], dtype=torch.int32, device="cuda"))
    assert bool((pool[7000] == 1).all()) and bool((pool[8998] == 4).all())
    h.fork(torch.tensor([[0, 2]], dtype=torch.int32, device="cuda"))
    assert table[2].tolist()[:3] == [8999, 4096, 0] and bool((pool[0, :8] == 3).all())
    live = torch.zeros(1, dtype=torch.int32, device="cuda")
    h.compact(live_out=live)
    # pages 0 and 5 stay below 5 live ones only where 0; 5, 4096, 8191, 8999 move to 1, 2, 3, 4
    assert int(live) == 5 and int(h.status_flag) == 0
    assert table.tolist() == [[4, 2, 3, 0], [1, 0, 0, 0], [4, 2, 0, 0]]
    assert [bool((pool[p] == x).all()) for p, x in ((1, 4), (2, 2), (3, 3), (4, 1))] == [True] * 4
    del pool, h
    torch.cuda.empty_cache()
