"""Rows that have grown past the length that the splits were planned for: every token is still attended."""
import numpy as np
import pytest

from oracle import paged_decode_oracle as O
from oracle import q4_cache_oracle as Q
from paper_2606_07665_b200 import workloads as W
from tests.test_gpu_parity import check_out
from tests.test_gpu_q4 import Case, bits, check, dev, f64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rt():
    import torch
    from paper_2606_07665_b200 import binding, build, runner
    build.build()
    binding.ac_init(0)
    torch.cuda.set_device(0)
    return runner


# (window, sinks): the last one's span is longer than the plan, so a plan that is too short cuts it too
MASKS = [(0, 0), (40, 6), (2000, 0), (2000, 9)]
SPLITS = [1, 2, 5]


@pytest.mark.parametrize("window,sinks", MASKS)
@pytest.mark.parametrize("splits", SPLITS)
def test_q4_rows_past_the_plan(rt, window, sinks, splits):
    import torch
    planned = np.array([63, 10, -1, 127], dtype=np.int32)
    c = Case(rt, 60, [64, 1500, -1, 700], 8, 2, 64, 16, 32)
    h = rt.Q4DecodeStep(c.upload(rt), dev(c.table), dev(c.lens), 8, lens_host=planned, window=window, sinks=sinks, num_splits=splits)
    q = bits(c.rng, 4, 8, 64)
    out = h.attention(dev(q))
    torch.cuda.synchronize()
    ref, room = Q.attention(q, c.fetch, np.where(c.lens >= 0, c.lens + 1, 0), 2, window, sinks, slack=True)
    check(f64(out), ref, room, f"splits {splits}")


@pytest.mark.parametrize("window,sinks", MASKS)
@pytest.mark.parametrize("splits", SPLITS)
@pytest.mark.parametrize("d", [128, 64])
def test_bf16_rows_past_the_plan(rt, window, sinks, splits, d):
    import torch
    w = W.make_workload("past", 61, B=4, Hq=8, Hkv=2, d=d, page_size=16, num_pages=160, context_lens=[64, 1500, 3, 700], rope_base=10000.0,
                        inactive_rows=(2,))
    q_rot, k_after, v_after = O.oracle_rope_kv_append(w.q, w.k_new, w.v_new, w.k_cache, w.v_cache, w.block_table, w.context_lens,
                                                      w.rope_cos, w.rope_sin, w.page_size)

    def fetch(b, h, t):
        pg, sl = w.block_table[b, t // w.page_size], t % w.page_size
        return O.bf16_to_f64(k_after[pg, sl, h]), O.bf16_to_f64(v_after[pg, sl, h]), np.zeros((len(t), w.d))

    ref = Q.attention(q_rot, fetch, np.where(w.context_lens >= 0, w.context_lens + 1, 0), w.Hkv, window, sinks)
    h = rt.PagedAttention(dev(k_after), dev(v_after), dev(w.block_table), dev(w.context_lens), 8, lens_host=[63, 10, -1, 127], window=window,
                          sinks=sinks, num_splits=splits)
    out = h.attention(dev(q_rot))
    torch.cuda.synchronize()
    check_out(f64(out), ref, f"splits {splits}")
    # and with the merge as a launch of its own
    st = rt.DecodeStep(w, num_splits=splits, max_context_len=128, fused_merge=False, window=window, sinks=sinks)
    st.step()
    torch.cuda.synchronize()
    check_out(st.out_f64(), ref, f"separate merge, splits {splits}")


def test_steps_past_the_plan(rt):
    # a row whose length fills the grid exactly, then two steps more: the token just appended counts
    import torch
    c = Case(rt, 62, [127, 20], 4, 2, 64, 16, 64, room=4)
    cos, sin = W.rope_table(256, 64, 10000.0)
    lens = dev(c.lens)
    cache = c.upload(rt)
    table = dev(c.table)
    h = rt.Q4DecodeStep(cache, table, lens, 4, lens_host=c.lens, num_splits=1, rope_cos=dev(cos), rope_sin=dev(sin))
    wide = rt.Q4DecodeStep(cache, table, lens, 4, max_context_len=512, num_splits=1)
    for _ in range(3):
        q, k, v = (dev(bits(c.rng, 2, n, 64)) for n in (4, 2, 2))
        q_rot = h.append(q, k, v)
        assert torch.equal(h.attention(q_rot), wide.attention(q_rot))
        lens.add_(1)
