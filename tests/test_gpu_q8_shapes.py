"""8-bit attention and the steps around it in every shape of the kernel's CTA: grids of few and of many CTAs, short and long splits."""
import numpy as np
import pytest

from oracle import q8_cache_oracle as Q
from paper_2606_07665_b200 import workloads as W
from tests.test_gpu_q8 import Case, bits, dev, run_attention

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rt():
    import torch
    from paper_2606_07665_b200 import build, runner
    build.build()
    torch.cuda.set_device(0)
    return runner


class Drawn(Case):
    """A case whose codes are drawn from a few thousand rounded normal values instead of being rounded one by one."""

    def __init__(self, seed, lens, Hq, Hkv, d, ps, block, fmt, layout="token_major", room=1, spare=3, exponents=(-6, -3)):
        super().__init__(seed, [-1] * len(lens), Hq, Hkv, d, ps, block, fmt, layout, room=0, spare=spare)
        rng = self.rng
        self.lens = np.asarray(lens, dtype=np.int32)
        need = np.array([-(-(int(n) + room) // ps) for n in lens])
        self.num_pages = int(need.sum()) + spare
        perm = rng.permutation(self.num_pages)
        self.table = np.full((self.B, int(need.max()) + 1), -7, dtype=np.int32)
        some = Q.encode(rng.standard_normal(8192) * (32.0 if fmt == Q.INT8 else 64.0), fmt)
        k, v = (some[rng.integers(0, len(some), (self.num_pages, ps, Hkv, d))] for _ in range(2))
        scales = np.ldexp(np.float32(1), rng.integers(*exponents, (self.num_pages, Hkv, ps // block, 2))).astype(np.float32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = perm[at:at + n]
            at += n
            tokens = int(lens[b]) + room
            last, slot = self.table[b, n - 1], (tokens - 1) % ps
            for pool in (k, v):
                pool[last, slot + 1:] = 0x7F
            scales[last, :, slot // block + 1:] = np.nan
        for pool in (k, v):
            pool[perm[at:]] = 0x7F
        scales[perm[at:]] = np.nan
        self.cache = Q.Cache(k, v, scales, fmt)


def shape(ctas, split_tokens, wide, sms):
    """(warps, CTAs per SM) that the grid gets."""
    if ctas <= sms:
        return 8, 1
    if ctas <= 2 * sms or split_tokens > 2560:
        return (6 if wide else 4), 2
    return (3, 4) if ctas > 4 * sms and not wide else (4, 3)


# grid in CTAs per SM, the longest context that the plan allows for, the shape for groups of at most eight heads
GRIDS = [(1.3, 700, (4, 2)), (2.7, 3000, (4, 2)), (2.7, 700, (4, 3)), (4.3, 700, (3, 4))]


def drawn(rt, seed, per_sm, longest, Hkv, group, d, ps, block, fmt, splits):
    import torch
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    B = -(-int(per_sm * sms) // (Hkv * splits))
    rng = np.random.default_rng(seed)
    lens = rng.integers(0, 90, B)
    lens[:8] = 0, 15, 16, 31, longest - 1, longest // 2, 63, longest // 3
    return Drawn(seed, lens[rng.permutation(B)], group * Hkv, Hkv, d, ps, block, fmt), B * Hkv * splits, sms


@pytest.mark.parametrize("per_sm,longest,want", GRIDS)
@pytest.mark.parametrize("fmt,group", [(Q.INT8, 4), (Q.E4M3, 4), (Q.INT8, 16), (Q.E4M3, 9), (Q.INT8, 1), (Q.E4M3, 8)])
@pytest.mark.parametrize("d,ps,block", [(128, 16, 16), (64, 64, 32)])
@pytest.mark.parametrize("splits", [1, 3])
@pytest.mark.parametrize("windowed", [False, True])
def test_attention(rt, per_sm, longest, want, fmt, group, d, ps, block, splits, windowed):
    window, sinks = 0, 0
    if windowed:
        window, sinks = (2700 if longest > 2560 else 130), 21
    span = min(longest, window + sinks + 64) if window else longest
    if longest > 2560 and splits > 1:
        longest, span = splits * longest, splits * span             # splits of more than 2560 tokens
        window = window and splits * window
    c, ctas, sms = drawn(rt, 50 + splits, per_sm, longest, 8, group, d, ps, block, fmt, splits)
    tokens = -(-span // splits)
    got = shape(ctas, tokens, group > 8, sms)
    if group <= 8:
        assert got == want
    run_attention(rt, c, window=window, sinks=sinks, splits=splits, max_context_len=longest)


@pytest.mark.parametrize("per_sm,longest,want", GRIDS)
@pytest.mark.parametrize("fmt,d,group", [(Q.E4M3, 128, 4), (Q.INT8, 64, 4), (Q.INT8, 128, 12)])
@pytest.mark.parametrize("splits", [1, 2])
def test_steps_back_to_back(rt, per_sm, longest, want, fmt, d, group, splits):
    """The bits of steps with a synchronisation after every call, with scales that grow at nearly every token; captured steps too."""
    import torch
    steps, Hkv, ps, block = 20, 4, 64, 32
    c, _, _ = drawn(rt, 60, per_sm, longest, Hkv, group, d, ps, block, fmt, splits)
    c = Drawn(61, c.lens, c.Hq, Hkv, d, ps, block, fmt, room=steps)
    cos, sin = W.rope_table(int(c.lens.max()) + steps, d, 10000.0)
    grow = torch.pow(1.5, torch.arange(steps, device="cuda") - 10.0)[:, None, None, None].bfloat16()
    q = dev(bits(c.rng, steps, c.B, c.Hq, d)).view(torch.bfloat16)
    k, v = (dev(bits(c.rng, steps, c.B, Hkv, d)).view(torch.bfloat16) * grow for _ in range(2))
    results = []
    for how in ("wait", "run", "graph"):
        cache, lens = c.upload(rt), dev(c.lens)
        step = rt.Q8DecodeStep(cache, dev(c.table), lens, c.Hq, max_context_len=longest, num_splits=splits, rope_cos=dev(cos), rope_sin=dev(sin))
        out = torch.zeros_like(q)
        q_in, k_new, v_new, q_rot, o = (torch.zeros_like(t[0]) for t in (q, k, v, q, q))
        torch.cuda.synchronize()
        if how == "graph":
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step.step(q_in, k_new, v_new, q_rot, o)
        for i in range(steps):
            if how == "graph":
                q_in.copy_(q[i]), k_new.copy_(k[i]), v_new.copy_(v[i])
                graph.replay()
                out[i].copy_(o)
            else:
                rot = step.append(q[i], k[i], v[i])
                if how == "wait":
                    torch.cuda.synchronize()
                step.attention(rot, out=out[i])
                if how == "wait":
                    torch.cuda.synchronize()
            lens += 1
        torch.cuda.synchronize()
        assert int(step.status_flag) == 0
        results.append((out, cache.k_codes, cache.v_codes, cache.scales))
    for other in results[1:]:
        for a, b in zip(results[0], other):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    assert torch.isfinite(results[0][0]).all()
