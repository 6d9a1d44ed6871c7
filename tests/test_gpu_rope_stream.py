"""Rotary rows of calls large enough for the streaming kernel: its border, positions past the table, tokens that stay as they are."""
import numpy as np
import pytest

from oracle import paged_decode_oracle as O
from tests.test_gpu_rope_rows import bits, dev, host

pytestmark = pytest.mark.gpu

BORDER = 24 << 20                                                   # bytes of q and k together


@pytest.fixture(scope="module")
def rt():
    import torch
    from paper_2606_07665_b200 import build, runner
    build.build()
    torch.cuda.set_device(0)
    return runner


def batch(rng, T, table, norms=None):
    """Ragged rows over T tokens, five of no row at either end; one row empty, one inactive, one past the table by all but ten tokens and
    one whose first token already is."""
    cut = np.sort(rng.choice(np.arange(200, T - 200, 100), 40, replace=False))      # rows of 100 tokens at least
    off = np.concatenate([[5], cut, cut[-1:], [T - 5]]).astype(np.int32)
    start = rng.integers(0, 50, len(off) - 1).astype(np.int32)
    start[7], start[20], start[25] = -1, table - 10, table
    return off, start


def places(off, start, T, table):
    """Position of every token, -1 where it has none."""
    pos = np.full(T, -1)
    for b, s in enumerate(start):
        if s >= 0:
            p = s + np.arange(off[b + 1] - off[b])
            pos[off[b]:off[b + 1]] = np.where(p < table, p, -1)
    return pos


@pytest.mark.parametrize("d,Hq,Hkv,R,interleaved,norm,beside", [(128, 17, 1, 128, False, False, 0), (128, 17, 3, 64, True, False, 6000), (64, 33, 5, 32, False, True, 0),
                                                                (64, 40, 0, 64, True, True, 0), (128, 7, 7, 16, False, True, 0),
                                                                (128, 12, 4, 128, False, False, -1), (64, 24, 8, 64, False, True, -1)])
def test_sampled_tokens_are_the_oracle_s(rt, d, Hq, Hkv, R, interleaved, norm, beside):
    """As many tokens as reach the border just, some more, and (`beside` -1) one token fewer, which the other kernel takes."""
    import torch
    from paper_2606_07665_b200 import binding as ac
    per_token = (Hq + Hkv) * d * 2
    T = -(-BORDER // per_token) + beside
    assert (T * per_token >= BORDER) == (beside >= 0)
    table = 5000 + T
    rng = np.random.default_rng(d + Hq)
    off, start = batch(rng, T, table)
    pos = places(off, start, T, table)
    w = (bits(rng, d), bits(rng, d)) if norm else (None, None)
    rope = rt.Rope.scaled(table, R, interleaved=interleaved, norm_eps=1e-5, q_norm_weight=dev(w[0]).view(torch.bfloat16) if norm else None,
                          k_norm_weight=dev(w[1]).view(torch.bfloat16) if norm else None)
    cos, sin = rope.cos.cpu().numpy(), rope.sin.cpu().numpy()
    joint = dev(bits(rng, T, Hq + Hkv + 1, d))
    q, k = joint[:, :Hq], joint[:, Hq:Hq + Hkv] if Hkv else None
    before = joint.clone()
    q_out, k_out = dev(bits(rng, T, Hq, d)), dev(bits(rng, T, Hkv, d)) if Hkv else None
    had = [t.clone() if t is not None else None for t in (q_out, k_out)]
    rope.rows(q, k, dev(start), dev(off), q_out=q_out, k_out=k_out)
    torch.cuda.synchronize()
    assert int(rope.status_flag) == ac.AC_FLAG_POSITION_OOB
    assert torch.equal(joint, before)
    still = torch.from_numpy(pos < 0).cuda()
    assert int(still.sum()) > 200                                   # of no row, inactive and past the table
    edges = np.concatenate([off[:-1], off[1:] - 1, [0, T - 1, off[20] + 9, off[20] + 10]])
    some = np.unique(np.concatenate([edges, rng.integers(0, T, 60)]))
    some = some[pos[some] >= 0]
    for x, out, was, wt in ((q, q_out, had[0], w[0]), (k, k_out, had[1], w[1])):
        if x is None:
            continue
        assert torch.equal(out[still], was[still])
        picked = torch.from_numpy(some).cuda()
        given, got = host(x[picked]), host(out[picked])
        for i, t in enumerate(some):
            for h in range(0, x.shape[1], 3):
                y = given[i, h] if wt is None else O.rms_norm_bf16(given[i, h], wt, 1e-5)
                assert np.array_equal(got[i, h], O.rope_rotate_variant_bf16(y, cos[pos[t]], sin[pos[t]], R, interleaved)), (t, h)
    rope.rows(q, k, dev(start), dev(off), q_out=q, k_out=k)         # in place, in the joint tensor
    for x, out, at in ((q, q_out, slice(0, Hq)), (k, k_out, slice(Hq, Hq + Hkv))):
        if x is not None:
            assert torch.equal(x[~still], out[~still]) and torch.equal(x[still], before[:, at][still])
    assert torch.equal(joint[:, Hq + Hkv:], before[:, Hq + Hkv:])


def test_calls_past_the_table_alone_set_the_status(rt):
    """No token of the call has a position: nothing is written, and the status says so."""
    import torch
    from paper_2606_07665_b200 import binding as ac
    rope = rt.Rope.scaled(16, 128)
    q = torch.randn(4000, 32, 128, device="cuda").bfloat16()
    was = q.clone()
    rope.rows(q, None, dev(np.array([16], np.int32)), dev(np.array([0, 4000], np.int32)), q_out=q)
    torch.cuda.synchronize()
    assert int(rope.status_flag) == ac.AC_FLAG_POSITION_OOB and torch.equal(q, was)


@pytest.mark.parametrize("positions,half", [(4, 9), (1000, 32), (131, 64), (70001, 20), (8193, 64)])
def test_tables_in_a_larger_buffer(rt, positions, half):
    """Nothing in front of the tables or behind them is written; counts that are no multiple of a thread's run among them."""
    import torch
    n = positions * half
    big = torch.full((2, 64 + n + 64), 7.0, device="cuda")
    apart = torch.full((64 + n + 64 + 3,), 7.0, device="cuda")
    cos, sin = big[0, 64:64 + n].view(positions, half), apart[64:64 + n].view(positions, half)
    rt.Rope(cos, sin).fill(3, base=1e6)
    torch.cuda.synchronize()
    assert (big[0, :64] == 7).all() and (big[0, 64 + n:] == 7).all() and (big[1] == 7).all()
    assert (apart[:64] == 7).all() and (apart[64 + n:] == 7).all()
    assert (cos.abs() <= 1).all() and (sin.abs() <= 1).all()
