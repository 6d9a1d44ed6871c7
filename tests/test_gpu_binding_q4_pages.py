"""The binding's functions of the 4-bit cache and of the pages, one after another as a caller without the runner's objects uses
them; the same calls through those objects give the same bits."""
import numpy as np
import pytest

from paper_2606_07665_b200 import workloads as W
from tests.test_gpu_cache_pages import i32
from tests.test_gpu_q4 import bits, dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rt():
    import torch
    from paper_2606_07665_b200 import binding, build, runner
    build.build()
    binding.ac_init(0)
    torch.cuda.set_device(0)
    return runner


def test_store_append_attend_fork_release_compact(rt):
    import torch
    from paper_2606_07665_b200 import binding as ac
    rng = np.random.default_rng(110)
    B, Hq, Hkv, d, ps, group, num_pages, width = 4, 8, 2, 128, 16, 64, 60, 6
    cos, sin = (dev(x) for x in W.rope_table(96, d, 10000.0))
    off, start = i32([0, 20, 53, 58, 58]), i32([0] * B)
    k, v = dev(bits(rng, 58, Hkv, d)), dev(bits(rng, 58, Hkv, d))
    q, k_new, v_new = (dev(bits(rng, B, n, d)) for n in (Hq, Hkv, Hkv))
    weight = dev(bits(rng, d))
    pairs, gone = i32([[1, 3]]), i32([0])
    shape = (B, Hq, Hkv, d, ps, num_pages)

    def state():
        cache = rt.Q4Cache.empty(num_pages, ps, Hkv, d, group)
        lens = i32([0, 0, 0, -1])
        table, refs = i32(np.zeros((B, width), np.int32).tolist()), i32([1, 0, 1] + [0] * (num_pages - 3))
        return cache, table, lens, refs

    def everything(cache, table, lens, refs, *more):
        torch.cuda.synchronize()
        return [x.clone() for x in (cache.k_codes, cache.v_codes, cache.params, table, lens, refs, *more)]

    # through the objects
    cache, table, lens, refs = state()
    pages = rt.CachePages(cache.pools, table, lens, refs, ps)
    pages.reserve(33)
    cache.store(k, v, table, start, off)
    kb, vb = cache.load(table, start, off, 58)
    lens[:3] = i32([20, 33, 5])
    pages.trim()
    pages.fork(pairs)
    pages.reserve(1)
    step = rt.Q4DecodeStep(cache, table, lens, Hq, max_context_len=96, num_splits=3, window=30, sinks=3, rope_cos=cos, rope_sin=sin, row_order=[2, 0, 3, 1],
                           rope_variants=dict(q_norm_weight=weight, norm_eps=1e-5, interleaved=True))
    q_rot = step.append(q, k_new, v_new)
    out = step.attention(q_rot)
    lens.add_((lens >= 0).int())
    pages.release(gone)
    pages.compact()
    pages.copy(i32([[0, 59], [1, 58]]))
    want = everything(cache, table, lens, refs, kb, vb, q_rot, out)
    assert int(pages.status_flag) == int(step.status_flag) == int(cache.status_flag) == 0

    # through the binding
    cache, table, lens, refs = state()
    flag = i32([0])
    c = ac.q4_cache(cache.k_codes, cache.v_codes, cache.params, *(cache.k_codes.stride(i) for i in (0, 1, 2)), group)
    pools = ac.page_pools([(cache.k_codes, ps * Hkv * d // 2, 1), (cache.v_codes, ps * Hkv * d // 2, 1), (cache.params, ps * Hkv * 8 * (d // group), Hkv)])
    room = torch.empty(ac.ac_cache_workspace_bytes(B, num_pages, 1), dtype=torch.uint8, device="cuda")
    kb, vb, q_rot, out = (torch.zeros_like(x) for x in (k, v, q, q))
    ac.ac_cache_reserve(table, width, lens, refs, 33, B, ps, num_pages, room, room.numel(), flag)
    ac.ac_kv_store_q4(k, v, c, table, width, start, off, 58, B, Hkv, d, ps, num_pages, flag)
    ac.ac_kv_load_q4(kb, vb, c, table, width, start, off, 58, B, Hkv, d, ps, num_pages, flag)
    lens[:3] = i32([20, 33, 5])
    ac.ac_cache_trim(table, width, lens, refs, B, ps, num_pages, flag)
    ac.ac_cache_fork(pools, 3, table, width, lens, refs, pairs, 1, B, ps, num_pages, room, room.numel(), flag)
    ac.ac_cache_reserve(table, width, lens, refs, 1, B, ps, num_pages, room, room.numel(), flag)
    ac.ac_rope_kv_append_q4(q, q_rot, k_new, v_new, c, table, width, lens, cos, sin, 96, *shape, flag, q_norm_weight=weight, norm_eps=1e-5, interleaved=True)
    n = ac.ac_fused_workspace_bytes(B, Hq, Hkv, d, 3)
    workspace = torch.zeros(n, dtype=torch.uint8, device="cuda")
    ac.ac_paged_decode_attn_q4(q_rot, c, table, width, lens, 1, 0.0, 3, workspace, n, out, *shape, 96, flag, window=30, sinks=3, row_order=i32([2, 0, 3, 1]))
    lens.add_((lens >= 0).int())
    ac.ac_cache_release(table, width, lens, refs, gone, 1, B, ps, num_pages, flag)
    ac.ac_cache_compact(pools, 3, table, table, width, lens, refs, refs, B, ps, num_pages, None, room, room.numel(), flag)
    ac.ac_cache_copy_pages(pools, 3, i32([[0, 59], [1, 58]]), 2, num_pages, flag)
    got = everything(cache, table, lens, refs, kb, vb, q_rot, out)
    assert int(flag) == 0
    for i, (a, b) in enumerate(zip(got, want)):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), i
    with pytest.raises(ac.AcError):
        ac.ac_paged_decode_attn_q4(q_rot, c, table, width, lens, 1, 0.0, 3, workspace, n - 1, out, *shape, 96)
