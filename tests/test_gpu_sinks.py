"""The sliding window with sinks over the bf16 cache, in every launch flavour, against the oracle."""
import numpy as np
import pytest

from oracle import paged_decode_oracle as O
from oracle import q4_cache_oracle as Q
from paper_2606_07665_b200 import workloads as W
from tests.test_gpu_parity import check_out

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rt():
    import torch
    from paper_2606_07665_b200 import binding, build, runner
    build.build()
    binding.ac_init(0)
    torch.cuda.set_device(0)
    return runner


def reference(w, window, sinks):
    q_rot, k_after, v_after = O.oracle_rope_kv_append(w.q, w.k_new, w.v_new, w.k_cache, w.v_cache, w.block_table, w.context_lens,
                                                      w.rope_cos, w.rope_sin, w.page_size)

    def fetch(b, h, t):
        pg, sl = w.block_table[b, t // w.page_size], t % w.page_size
        return O.bf16_to_f64(k_after[pg, sl, h]), O.bf16_to_f64(v_after[pg, sl, h]), np.zeros((len(t), w.d))

    n = np.where(w.context_lens >= 0, w.context_lens + 1, 0)
    return q_rot, k_after, v_after, Q.attention(q_rot, fetch, n, w.Hkv, window, sinks)


def poison(w, window, sinks):
    """Every cached token that is not attended becomes NaN."""
    for b in range(w.B):
        n = int(w.context_lens[b]) + 1
        seen = np.isin(np.arange(max(n - 1, 0)), Q.visible(n, window, sinks))
        for t in np.nonzero(~seen)[0]:
            w.k_cache[w.block_table[b, t // w.page_size], t % w.page_size] = W.BF16_NAN
            w.v_cache[w.block_table[b, t // w.page_size], t % w.page_size] = W.BF16_NAN


def run(rt, w, window, sinks, splits, fused, layout="token_major"):
    import torch
    poison(w, window, sinks)
    q_rot, k_after, v_after, ref = reference(w, window, sinks)
    st = rt.DecodeStep(w, num_splits=splits, layout=layout, fused_merge=bool(fused), fused_step=fused == "step", window=window, sinks=sinks)
    st.step()
    torch.cuda.synchronize()
    assert int(st.status_flag) == 0
    assert np.array_equal(rt.bits_of(st.q_rot), q_rot)
    k, v = st.cache_bits()
    assert np.array_equal(k, k_after) and np.array_equal(v, v_after)
    check_out(st.out_f64(), ref, f"window {window} sinks {sinks} splits {splits} {fused}")
    return st


@pytest.mark.parametrize("fused", [False, True, "step"])
@pytest.mark.parametrize("window,sinks,splits", [(1, 1, 1), (7, 4, 1), (16, 16, 2), (33, 100, 1), (100, 5, 3), (300, 64, 2), (5000, 3, 2),
                                                 (150, 470, 3), (150, 490, 1), (64, 2**31 - 1, 2), (2**31 - 1, 5, 1)])
@pytest.mark.parametrize("d,ps", [(128, 16), (64, 80)])
def test_sinks(rt, window, sinks, splits, fused, d, ps):
    w = W.make_workload("sinks", 71, B=6, Hq=8, Hkv=2, d=d, page_size=ps, num_pages=150, context_lens=[0, 5, 100, 640, 9, 627],
                        rope_base=10000.0, inactive_rows=(4,))
    run(rt, w, window, sinks, splits, fused)


@pytest.mark.parametrize("B,Hq,Hkv,lens,window,sinks,splits,fused", [
    (1, 32, 8, [20000], 1024, 4, None, True),                # one long row: splits, twelve warps
    (1, 32, 8, [6000], 1024, 4, None, "step"),
    (2, 32, 2, [3000, 70], 500, 37, 4, True),                # sixteen heads per KV head, merge in a cluster
    (40, 8, 8, [900 + 17 * i for i in range(40)], 256, 20, 1, "step"),   # more than one CTA per SM
    (20, 16, 8, [5000] * 20, 4096, 100, None, True),         # one wave of long splits: four warps
])
def test_sinks_launch_shapes(rt, B, Hq, Hkv, lens, window, sinks, splits, fused):
    pages = sum(n // 16 + 1 for n in lens) + 2
    w = W.make_workload("sinks", 72, B=B, Hq=Hq, Hkv=Hkv, d=128, page_size=16, num_pages=pages, context_lens=lens, rope_base=10000.0)
    run(rt, w, window, sinks, splits, fused, layout="head_major")


def test_no_window_ignores_sinks_and_no_sinks_is_the_window(rt):
    import torch
    w = W.make_workload("sinks", 73, B=3, Hq=8, Hkv=2, d=128, page_size=16, num_pages=96, context_lens=[200, 37, 333], rope_base=10000.0)
    outs = []
    for window, sinks in ((0, 0), (0, 9), (50, 0)):
        st = rt.DecodeStep(w, num_splits=2, window=window, sinks=sinks)
        st.step()
        torch.cuda.synchronize()
        outs.append(st.out_f64())
    assert np.array_equal(outs[0], outs[1])
    check_out(outs[2], O.oracle_decode_step(w, window=50)[3], "window alone")


def test_paged_attention_object(rt):
    import torch
    w = W.make_workload("sinks", 74, B=4, Hq=12, Hkv=3, d=64, page_size=32, num_pages=80, context_lens=[300, 31, 0, 500], rope_base=10000.0,
                        inactive_rows=(2,))
    for layout in ("token_major", "head_major"):
        q_rot, k_after, v_after, ref = reference(w, 70, 10)
        move = (lambda x: x) if layout == "token_major" else (lambda x: np.ascontiguousarray(x.transpose(0, 2, 1, 3)))
        up = lambda x: torch.from_numpy(x.view(np.int16) if x.dtype == np.uint16 else x).cuda()              # noqa: E731
        h = rt.PagedAttention(up(move(k_after)), up(move(v_after)), up(w.block_table), up(w.context_lens), 12, lens_host=w.context_lens,
                              window=70, sinks=10, layout=layout)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            out = h.attention(up(q_rot))
        torch.cuda.synchronize()
        check_out(O.bf16_to_f64(rt.bits_of(out)), ref, layout)
