"""What is measured of the 8-bit paged cache and of rotary positions for prompts and long contexts.

Every case is a plain dict; ``run`` makes one pass through an operator, either in its plain form (elementary torch
operations in 32 or 64 bits) or, with ``own`` set, by the calls a serving program makes.

Kinds of cases
  append   RoPE of the new q and k, the new k and v quantised into their 8-bit blocks, and the written blocks read back
  store    pieces of prompts quantised into the 8-bit pages behind what the rows hold, and read back
  attn     decode attention over the 8-bit cache, optionally with a window and sinks
  rope     the queries and keys of a batch of prompts rotated: half or interleaved pairs, all or part of the head
  table    cosines and sines of scaled rotary frequencies for a range of positions

The 8-bit format: a block of ``block`` consecutive slots of a page, for one head and one of K and V, has a scale 2^e; e is
the least one with max |x| <= M 2^e over what the block holds (M = 127 for int8, 448 for e4m3; -100 <= e <= 121, 119), a
code is x / 2^e rounded to the format, and stands for code * 2^e.  A block that is written on keeps its scale or, where the
new tokens need a larger one, has the codes that it holds rounded again under that.
"""
import math

import numpy as np
import torch

own = False

_DEV = "cuda"
_LARGEST = {"int8": 127.0, "e4m3": 448.0}
_TOP = {"int8": 121, "e4m3": 119}


def listed():
    return [
        # one token of each of 8 requests, the middle bucket of the graph sweep: latency of a short step
        dict(name="append_b8", kind="append", fmt="e4m3", block=32, B=8, Hq=28, Hkv=4, d=128, ps=32, lo=512, hi=2048, rotary=128, pairs="half", norm=False, len_seed=51),
        # the largest bucket of the same sweep, rotary on half of the head in interleaved pairs
        dict(name="append_b256", kind="append", fmt="int8", block=16, B=256, Hq=28, Hkv=4, d=128, ps=32, lo=512, hi=2048, rotary=64, pairs="interleaved", norm=False, len_seed=54),
        # the next pieces of four prompts that are fed in turns, behind what the cache holds
        dict(name="store_pieces", kind="store", fmt="e4m3", block=16, B=4, Hq=8, Hkv=8, d=128, ps=16, start=777, lo=1, hi=200, len_seed=21),
        # 32 prompts of up to 4096 tokens entering the cache together and read back for a prefix
        dict(name="store_b32", kind="store", fmt="int8", block=16, B=32, Hq=32, Hkv=8, d=128, ps=16, start=0, lo=17, hi=4096, len_seed=7),
        # the smallest decode step: 512 tokens, two KV heads of 64 elements
        dict(name="attn_tiny", kind="attn", fmt="int8", block=16, B=1, Hq=8, Hkv=2, d=64, ps=16, lo=512, hi=512, len_seed=1, window=0, sinks=0),
        # continuous batching: 64 requests of 128 to 8192 tokens
        dict(name="attn_b64", kind="attn", fmt="e4m3", block=16, B=64, Hq=32, Hkv=8, d=128, ps=16, lo=128, hi=8192, len_seed=3, window=0, sinks=0),
        # sixteen query heads per KV head under a window that keeps the first tokens
        dict(name="attn_window_b32", kind="attn", fmt="int8", block=64, B=32, Hq=32, Hkv=2, d=128, ps=64, lo=2048, hi=12288, len_seed=6, window=4096, sinks=4),
        # long contexts, eight query heads per KV head
        dict(name="attn_long", kind="attn", fmt="e4m3", block=32, B=4, Hq=64, Hkv=8, d=128, ps=32, lo=131071, hi=131071, len_seed=4, window=0, sinks=0),
        # a short question behind a long conversation
        dict(name="rope_b1", kind="rope", B=1, Hq=28, Hkv=4, d=128, start=20000, lo=37, hi=37, rotary=128, pairs="half", norm=False, len_seed=5),
        # 32 prompts of up to 4096 tokens
        dict(name="rope_b32", kind="rope", B=32, Hq=32, Hkv=8, d=128, start=0, lo=17, hi=4096, rotary=128, pairs="half", norm=False, len_seed=7),
        # positions of a short context, half of the head rotated
        dict(name="table_4k", kind="table", first=0, positions=4096, rotary=64, base=10000.0, scaling="linear", factor=4.0),
        # the same model stretched to 131072 positions, low frequencies slowed down and high ones kept
        dict(name="table_128k", kind="table", first=0, positions=131072, rotary=128, base=500000.0, scaling="ramp", factor=32.0),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["append", "store", "attn", "attn", "attn", "rope", "table"])
    if kind == "table":
        rotary = 2 * rng.randrange(2, 65)
        return dict(kind=kind, first=rng.choice([0, 0, 1000, 900000]), positions=_log(rng, 1, 131072), rotary=rotary, base=rng.choice([10000.0, 500000.0, 1000000.0]),
                    scaling=rng.choice(["none", "linear", "base", "ramp"]), factor=rng.choice([1.5, 2.0, 8.0, 40.0]))
    c = dict(kind=kind, len_seed=rng.randrange(1 << 20))
    d, hkv = rng.choice([64, 128, 128]), rng.choice([1, 2, 3, 4, 8])
    c.update(d=d, Hkv=hkv, Hq=hkv * rng.choice([1, 2, 3, 4, 7, 8, 16]))
    if kind != "rope":
        c.update(fmt=rng.choice(["int8", "e4m3"]), ps=rng.choice([16, 32, 48, 64, 128]))
        c.update(block=rng.choice([n for n in (16, 32, 48, 64, 128) if c["ps"] % n == 0]))
    if kind in ("append", "rope"):
        c.update(rotary=rng.choice([d, d, d // 2, d // 4 + 2]), pairs=rng.choice(["half", "half", "interleaved"]), norm=rng.random() < 0.25)
    if kind == "append":
        c.update(B=_log(rng, 1, 256), lo=rng.choice([0, 1, 100]), hi=_log(rng, 128, 4096))
    elif kind == "store":
        c.update(B=_log(rng, 1, 32), start=rng.choice([0, 0, 1, 100, 1000]), hi=_log(rng, 32, 2048))
        c.update(lo=rng.choice([0, 1, 17]) if c["B"] > 4 else 1)
    elif kind == "rope":
        c.update(B=_log(rng, 1, 32), start=rng.choice([0, 0, 1, 100, 100000]), hi=_log(rng, 32, 1024))
        c.update(lo=rng.choice([0, 1, 17]) if c["B"] > 4 else 1)
    else:
        c.update(B=_log(rng, 1, 64))
        hi = _log(rng, 16, max(64, 262144 // c["B"]))
        w = rng.randrange(1, hi + 1)
        window = w if rng.random() < 0.4 else 0
        c.update(lo=rng.choice([0, 1, max(1, hi // 2)]), hi=hi, window=window, sinks=_log(rng, 1, 600) if window else 0)
    return c


def _lengths(c):
    return np.random.default_rng(c["len_seed"]).integers(c["lo"], c["hi"] + 1, size=c["B"]).astype(np.int64)


def _visible(c, n):
    """Tokens a row of n tokens attends over."""
    w, s = c["window"], c["sinks"]
    return n if w == 0 else np.minimum(n, w) + np.minimum(s, np.maximum(n - w, 0))


def work(c):
    k = c["kind"]
    if k == "table":
        return {"bytes": c["positions"] * c["rotary"] * 4, "flops": c["positions"] * c["rotary"] * 3}
    kv = c["Hkv"] * c["d"]
    n = _lengths(c)
    if k == "rope":
        t = int(n.sum())
        far = int(n.max()) if t else 0
        return {"bytes": t * 4 * (c["Hq"] + c["Hkv"]) * c["d"] + far * 4 * c["rotary"], "flops": t * 3 * (c["Hq"] + c["Hkv"]) * c["rotary"]}
    if k == "append":
        B, back = c["B"], int((n % c["block"] + 1).sum())
        return {"bytes": B * (4 * c["Hq"] * c["d"] + 4 * kv + 2 * kv + 16 * c["Hkv"]) + back * 6 * kv, "flops": B * 6 * (c["Hq"] + 2 * c["Hkv"]) * c["d"]}
    if k == "store":
        t = int(n.sum())
        return {"bytes": t * (8 * kv + 4 * kv) + (t // c["block"] + 1) * 16 * c["Hkv"], "flops": t * 8 * kv}
    t = int(_visible(c, n + 1).sum())
    return {"bytes": t * 2 * kv + t // c["block"] * 8 * c["Hkv"] + 4 * c["B"] * c["Hq"] * c["d"], "flops": 4 * t * c["Hq"] * c["d"]}


# ---- inputs -----------------------------------------------------------------------------------------------------


def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device=_DEV, dtype=torch.float32).to(torch.bfloat16)


def _table(gen, pages_per_row, num_pages, width):
    """Scattered pages for each row; unused entries name a page that no row has."""
    perm = torch.randperm(num_pages, generator=gen, device=_DEV).to(torch.int32)
    used = int(pages_per_row.sum())
    table = torch.full((len(pages_per_row), width), int(perm[used]) if used < num_pages else 0, dtype=torch.int32, device=_DEV)
    counts = torch.from_numpy(pages_per_row).to(_DEV)
    first = torch.cumsum(counts, 0) - counts
    at = torch.arange(width, device=_DEV)[None, :]
    keep = at < counts[:, None]
    table[keep] = perm[(first[:, None] + at)[keep]]
    return table, perm[:used].long()


def _angles(c, positions):
    i = np.arange(c["rotary"] // 2, dtype=np.float64)
    ang = np.arange(positions, dtype=np.float64)[:, None] * np.power(500000.0, -2.0 * i / c["rotary"])[None, :]
    return torch.from_numpy(np.cos(ang).astype(np.float32)).to(_DEV), torch.from_numpy(np.sin(ang).astype(np.float32)).to(_DEV)


def _pools(gen, c, num_pages, used):
    """Codes and scales of a cache of normal values; the scales of pages that no row holds are NaN."""
    codes = []
    for _ in range(2):
        x = torch.randn(num_pages, c["ps"], c["Hkv"], c["d"], generator=gen, device=_DEV)
        codes.append((x * 32.0).round().clamp(-127, 127).to(torch.int8) if c["fmt"] == "int8" else (x * 64.0).to(torch.float8_e4m3fn))
    # pages begin at multiples of 16 bytes, whatever heads and blocks there are
    width = c["Hkv"] * (c["ps"] // c["block"]) * 2
    held = torch.full((num_pages, -(-width // 4) * 4), float("nan"), device=_DEV)
    scales = held[:, :width].view(num_pages, c["Hkv"], c["ps"] // c["block"], 2)
    e = torch.randint(-6, -3, (len(used), *scales.shape[1:]), generator=gen, device=_DEV)
    scales[used] = torch.ldexp(torch.ones_like(e, dtype=torch.float32), e)
    return codes[0], codes[1], scales


def _norm_weights(gen, c):
    return [(1.0 + 0.1 * torch.randn(c["d"], generator=gen, device=_DEV)).to(torch.bfloat16) for _ in range(2)] if c["norm"] else [None, None]


def prepare(case, seed):
    c = case
    gen = torch.Generator(device=_DEV).manual_seed(seed)
    st = {"case": c}
    if c["kind"] == "table":
        st["cos"], st["sin"] = (torch.zeros(c["positions"], c["rotary"] // 2, device=_DEV) for _ in range(2))
        # another seed stands for another stretch of the same context
        st["first"] = c["first"] + seed % 1000
        return st
    lens = _lengths(c)
    st["lens_host"], total = lens, int(lens.sum())
    if c["kind"] in ("store", "rope"):
        # rows are not all at the same place: each begins where its own conversation stands
        begin = c["start"] + np.arange(c["B"]) * (7 if c["start"] else 0)
        st["start"] = torch.from_numpy(begin.astype(np.int32)).to(_DEV)
        st["offsets"] = torch.from_numpy(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)).to(_DEV)
    if c["kind"] == "rope":
        # q and k as they leave a joint projection
        joint = _normal(gen, total, c["Hq"] + 2 * c["Hkv"], c["d"])
        st["q_in"], st["k_in"] = joint[:, :c["Hq"]], joint[:, c["Hq"]:c["Hq"] + c["Hkv"]]
        st["q_out"], st["k_out"] = (torch.zeros(total, h, c["d"], device=_DEV, dtype=torch.bfloat16) for h in (c["Hq"], c["Hkv"]))
        st["cos"], st["sin"] = _angles(c, int((begin + lens).max()) + 1)
        st["q_norm"], st["k_norm"] = _norm_weights(gen, c)
        return st
    tokens = begin + lens if c["kind"] == "store" else lens + 1
    need = -(-tokens // c["ps"])
    num_pages = int(need.sum() * 1.25) + 2
    st["table"], used = _table(gen, need, num_pages, max(1, int(need.max())))
    st["k"], st["v"], st["scales"] = _pools(gen, c, num_pages, used)
    st["num_pages"] = num_pages
    st["lens"] = torch.from_numpy(lens.astype(np.int32)).to(_DEV)
    if c["kind"] == "append":
        st["q_in"], st["k_new"], st["v_new"] = (_normal(gen, c["B"], h, c["d"]) for h in (c["Hq"], c["Hkv"], c["Hkv"]))
        st["q_out"] = torch.zeros_like(st["q_in"])
        st["cos"], st["sin"] = _angles(c, int(lens.max()) + 1)
        st["q_norm"], st["k_norm"] = _norm_weights(gen, c)
        # the block of each row that the new token belongs to is what is read back
        back = lens % c["block"] + 1
        st["start"] = torch.from_numpy((lens - lens % c["block"]).astype(np.int32)).to(_DEV)
        st["offsets"] = torch.from_numpy(np.concatenate([[0], np.cumsum(back)]).astype(np.int32)).to(_DEV)
        st["k_back"], st["v_back"] = (torch.zeros(int(back.sum()), c["Hkv"], c["d"], device=_DEV, dtype=torch.bfloat16) for _ in range(2))
    elif c["kind"] == "store":
        st["k_in"], st["v_in"] = (_normal(gen, total, c["Hkv"], c["d"]) for _ in range(2))
        # a few channels of the keys are much larger than the others
        st["k_in"][..., : c["d"] // 16] *= 8.0
        st["k_back"], st["v_back"] = torch.zeros_like(st["k_in"]), torch.zeros_like(st["v_in"])
    else:
        # slots behind a row's last token hold anything: here the codes that stand for no number, where there are any
        last, slot = torch.from_numpy(lens // c["ps"]).to(_DEV), torch.from_numpy(lens % c["ps"]).to(_DEV)
        page = st["table"][torch.arange(c["B"], device=_DEV), last].long()
        behind = torch.arange(c["ps"], device=_DEV)[None, :] > slot[:, None]
        for pool in (st["k"], st["v"]):
            raw = pool.view(torch.uint8)
            tail = raw[page]
            tail[behind] = 0x7F
            raw[page] = tail
        st["q"] = _normal(gen, c["B"], c["Hq"], c["d"])
        st["out"] = torch.zeros_like(st["q"])
    return st


# ---- the plain forms --------------------------------------------------------------------------------------------


def _to_bf16(x):
    """Nearest-even bf16 of 64-bit values, rounded once."""
    m, e = torch.frexp(x)
    return torch.ldexp(torch.round(m * 256.0), e - 8).to(torch.bfloat16)


def _code(y, fmt):
    """What the format holds of 32-bit values."""
    y = y.clamp(-_LARGEST[fmt], _LARGEST[fmt])
    return torch.round(y).to(torch.int8) if fmt == "int8" else y.to(torch.float8_e4m3fn)


def _write(st, page, slot, x, side):
    """Tokens x [n, heads, d] into their slots; the scales of the blocks that they begin or go on with follow."""
    c, scales, pool = st["case"], st["scales"][..., side], st["v"] if side else st["k"]
    pages, ps, nb = st["num_pages"], c["ps"], c["ps"] // c["block"]
    at = page * nb + slot // c["block"]
    most = torch.zeros(pages * nb, c["Hkv"], device=_DEV)
    most.scatter_reduce_(0, at[:, None].expand(-1, c["Hkv"]), x.float().abs().amax(-1), "amax")
    fresh = torch.zeros(pages * nb, dtype=torch.bool, device=_DEV)
    fresh[at[slot % c["block"] == 0]] = True
    touched = torch.zeros_like(fresh)
    touched[at] = True
    which = torch.nonzero(touched)[:, 0]
    m, e = torch.frexp(most[which].double() / _LARGEST[c["fmt"]])
    e = torch.where(m == 0.5, e - 1, e).clamp(-100, _TOP[c["fmt"]])
    e = torch.where(most[which] == 0, -100, e)
    need = torch.ldexp(torch.ones_like(m, dtype=torch.float32), e)
    held = scales[which // nb, :, which % nb]
    scale = torch.where(fresh[which][:, None], need, torch.maximum(held, need))
    blocks = pool.view(pages, nb, c["block"], c["Hkv"], c["d"])
    old = blocks[which // nb, which % nb].float()
    again = torch.where(fresh[which][:, None], 1.0, held / scale)[:, None, :, None]
    blocks[which // nb, which % nb] = _code(torch.nan_to_num(old * again), c["fmt"])
    scales[which // nb, :, which % nb] = scale
    pool[page, slot] = _code(x.float() / scales[page, :, slot // c["block"]][..., None], c["fmt"])


def _read(st, page, slot, side):
    c = st["case"]
    pool = st["v"] if side else st["k"]
    return (pool[page, slot].float() * st["scales"][page, :, slot // c["block"], side][..., None]).to(torch.bfloat16)


def _where(st, total):
    """Row, position, page and slot of the packed tokens."""
    c, off = st["case"], st["offsets"].long()
    t = torch.arange(total, device=_DEV)
    row = torch.searchsorted(off, t, right=True) - 1
    pos = t - off[row] + st["start"].long()[row]
    if "table" not in st:
        return pos, None, None
    return pos, st["table"][row, pos // c["ps"]].long(), pos % c["ps"]


def _rotate(c, x, cos, sin, weight):
    """x [n, heads, d] with the angles of its tokens, cos and sin [n, rotary / 2]."""
    y = x.double()
    if weight is not None:
        y = _to_bf16(y / torch.sqrt((y * y).mean(-1, keepdim=True) + 1e-6)).double()
        y = _to_bf16(y * weight.double()).double()
    r = c["rotary"]
    co, si = cos.double()[:, None], sin.double()[:, None]
    a, b = (y[..., 0:r:2], y[..., 1:r:2]) if c["pairs"] == "interleaved" else (y[..., : r // 2], y[..., r // 2:r])
    p, q = a * co - b * si, b * co + a * si
    turned = torch.stack((p, q), -1).flatten(-2) if c["pairs"] == "interleaved" else torch.cat((p, q), -1)
    return _to_bf16(torch.cat((turned, y[..., r:]), -1))


def _plain_append(st):
    c, pos = st["case"], st["lens"].long()
    cos, sin = st["cos"][pos], st["sin"][pos]
    page = st["table"].gather(1, (pos // c["ps"])[:, None])[:, 0].long()
    st["q_out"].copy_(_rotate(c, st["q_in"], cos, sin, st["q_norm"]))
    _write(st, page, pos % c["ps"], _rotate(c, st["k_new"], cos, sin, st["k_norm"]), 0)
    _write(st, page, pos % c["ps"], st["v_new"], 1)
    _, page, slot = _where(st, st["k_back"].shape[0])
    st["k_back"].copy_(_read(st, page, slot, 0))
    st["v_back"].copy_(_read(st, page, slot, 1))
    return st["q_out"], st["k_back"], st["v_back"]


def _plain_store(st):
    _, page, slot = _where(st, st["k_in"].shape[0])
    _write(st, page, slot, st["k_in"], 0)
    _write(st, page, slot, st["v_in"], 1)
    st["k_back"].copy_(_read(st, page, slot, 0))
    st["v_back"].copy_(_read(st, page, slot, 1))
    return st["k_back"], st["v_back"]


def _plain_attention(st):
    c = st["case"]
    n = st["lens"].long() + 1
    page = st["table"].long()
    t = torch.arange(page.shape[1] * c["ps"], device=_DEV)[None, :]
    seen = t < n[:, None]
    if c["window"]:
        seen = seen & ((t >= (n - c["window"])[:, None]) | (t < c["sinks"]))
    s = st["scales"][page].permute(0, 1, 3, 2, 4).repeat_interleave(c["block"], 2).flatten(1, 2)         # [B, tokens, head, side]
    k = torch.where(seen[:, :, None, None], st["k"][page].float().flatten(1, 2) * s[..., 0, None], 0.0)
    v = torch.where(seen[:, :, None, None], st["v"][page].float().flatten(1, 2) * s[..., 1, None], 0.0)
    q = st["q"].float().unflatten(1, (c["Hkv"], -1))
    s = torch.einsum("bhgd,bthd->bhgt", q, k) / math.sqrt(c["d"])
    s = torch.where(seen[:, None, None, :], s, float("-inf"))
    e = torch.exp(s - s.amax(-1, keepdim=True))
    o = torch.einsum("bhgt,bthd->bhgd", e / e.sum(-1, keepdim=True), v)
    st["out"].copy_(o.flatten(1, 2))
    return st["out"]


def _plain_rope(st):
    c = st["case"]
    pos, _, _ = _where(st, st["q_in"].shape[0])
    cos, sin = st["cos"][pos], st["sin"][pos]
    st["q_out"].copy_(_rotate(c, st["q_in"], cos, sin, st["q_norm"]))
    st["k_out"].copy_(_rotate(c, st["k_in"], cos, sin, st["k_norm"]))
    return st["q_out"], st["k_out"]


# a model trained on 8192 positions: frequencies that turn less than once in them are slowed down, more than four times kept
_RAMP = dict(original=8192, low=1.0, high=4.0)


def _magnitude(c):
    """Stretched tables also weigh the scores a little more."""
    return 0.1 * math.log(c["factor"]) + 1.0 if c["scaling"] == "ramp" else 1.0


def _plain_table(st):
    c = st["case"]
    r = c["rotary"]
    base = c["base"] * c["factor"] ** (r / (r - 2)) if c["scaling"] == "base" else c["base"]
    f = torch.pow(torch.tensor(base, dtype=torch.float64, device=_DEV), -2.0 * torch.arange(r // 2, dtype=torch.float64, device=_DEV) / r)
    if c["scaling"] == "linear":
        f = f / c["factor"]
    if c["scaling"] == "ramp":
        turns = _RAMP["original"] * f / (2.0 * math.pi)
        keep = ((turns - _RAMP["low"]) / (_RAMP["high"] - _RAMP["low"])).clamp(0.0, 1.0)
        f = keep * f + (1.0 - keep) * f / c["factor"]
    p = torch.arange(st["first"], st["first"] + c["positions"], dtype=torch.float64, device=_DEV)
    angle = p[:, None] * f[None, :]
    st["cos"].copy_(_magnitude(c) * torch.cos(angle))
    st["sin"].copy_(_magnitude(c) * torch.sin(angle))
    return st["cos"], st["sin"]


# ---- the framework's calls --------------------------------------------------------------------------------------


def _handle(st):
    """What a serving program keeps from step to step: the plan, the workspace and the objects that hold its buffers."""
    from paper_2606_07665_b200 import runner

    c = st["case"]
    if c["kind"] == "table":
        more = dict(original=_RAMP["original"], low=_RAMP["low"], high=_RAMP["high"], magnitude=_magnitude(c)) if c["scaling"] == "ramp" else {}
        return runner.Rope(st["cos"], st["sin"]), dict(base=c["base"], scaling=c["scaling"], factor=c["factor"], **more)
    variants = {}
    if c["kind"] in ("append", "rope"):
        variants = dict(rotary_dim=c["rotary"], interleaved=c["pairs"] == "interleaved", q_norm_weight=st["q_norm"], k_norm_weight=st["k_norm"], norm_eps=1e-6)
    if c["kind"] == "rope":
        return runner.Rope(st["cos"], st["sin"], **variants)
    cache = runner.Q8Cache(st["k"], st["v"], st["scales"])
    if c["kind"] == "store":
        return cache
    return runner.Q8DecodeStep(cache, st["table"], st["lens"], Hq=c["Hq"], lens_host=st["lens_host"], window=c.get("window", 0), sinks=c.get("sinks", 0), rope_cos=st.get("cos"),
                               rope_sin=st.get("sin"), rope_variants=variants)


def _own(st):
    kind = st["case"]["kind"]
    if "handle" not in st:
        st["handle"] = _handle(st)
    h = st["handle"]
    if kind == "append":
        h.append(st["q_in"], st["k_new"], st["v_new"], q_out=st["q_out"])
        h.cache.load(st["table"], st["start"], st["offsets"], k_out=st["k_back"], v_out=st["v_back"])
        return st["q_out"], st["k_back"], st["v_back"]
    if kind == "store":
        h.store(st["k_in"], st["v_in"], st["table"], st["start"], st["offsets"])
        h.load(st["table"], st["start"], st["offsets"], k_out=st["k_back"], v_out=st["v_back"])
        return st["k_back"], st["v_back"]
    if kind == "attn":
        h.attention(st["q"], out=st["out"])
        return st["out"]
    if kind == "rope":
        h.rows(st["q_in"], st["k_in"], st["start"], st["offsets"], q_out=st["q_out"], k_out=st["k_out"])
        return st["q_out"], st["k_out"]
    rope, how = h
    rope.fill(first_position=st["first"], **how)
    return st["cos"], st["sin"]


def run(state):
    if own:
        return _own(state)
    plain = {"append": _plain_append, "store": _plain_store, "attn": _plain_attention, "rope": _plain_rope, "table": _plain_table}
    return plain[state["case"]["kind"]](state)


# ---- 64 bits, from the definitions ------------------------------------------------------------------------------


def exact(case, seed):
    c = case
    st = prepare(case, seed)
    f64 = torch.float64

    if c["kind"] == "table":
        cos, sin = np.empty(st["cos"].shape), np.empty(st["sin"].shape)
        p = np.arange(st["first"], st["first"] + c["positions"], dtype=np.longdouble)
        for i in range(c["rotary"] // 2):
            b = np.longdouble(c["base"])
            if c["scaling"] == "base":
                b *= np.longdouble(c["factor"]) ** (np.longdouble(c["rotary"]) / (c["rotary"] - 2))
            f = b ** (np.longdouble(-2 * i) / c["rotary"])
            if c["scaling"] == "linear":
                f /= c["factor"]
            elif c["scaling"] == "ramp":
                turns = _RAMP["original"] * f / (2 * np.longdouble("3.14159265358979323846264338327950288"))
                if turns < _RAMP["low"]:
                    f /= c["factor"]
                elif turns <= _RAMP["high"]:
                    g = (turns - _RAMP["low"]) / (_RAMP["high"] - _RAMP["low"])
                    f = (1 - g) * f / c["factor"] + g * f
            m = 1 + 0.1 * math.log(c["factor"]) if c["scaling"] == "ramp" else 1.0
            cos[:, i], sin[:, i] = (m * np.cos(p * f)).astype(np.float64), (m * np.sin(p * f)).astype(np.float64)
        return torch.from_numpy(cos), torch.from_numpy(sin)

    def step(y):
        """Distance of the values that the format holds around y."""
        if c["fmt"] == "int8":
            return torch.ones_like(y)
        return torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)

    def rounded(y):
        s = step(y)
        return torch.clamp(torch.round(y / s) * s, -_LARGEST[c["fmt"]], _LARGEST[c["fmt"]])

    def through(x, held, before):
        """Block by block: tokens x [n, heads, d] behind `before` tokens of values held [before, heads, d] under their scale [heads]."""
        old, s_old = held
        most = x.to(f64).abs().amax((0, 2))
        s = torch.empty_like(most)
        for h in range(c["Hkv"]):
            e = -100
            while e < _TOP[c["fmt"]] and float(most[h]) > _LARGEST[c["fmt"]] * 2.0 ** e:
                e += 1
            s[h] = 2.0 ** e
        if before:
            s = torch.maximum(s, s_old)
        s = s[None, :, None]
        return torch.cat((rounded(old / s) * s, rounded(x.to(f64) / s) * s)) if before else rounded(x.to(f64) / s) * s

    def turned(x, positions, weight):
        """[n, heads, d] at the n positions."""
        y = x.to(f64)
        if weight is not None:
            y = y / torch.sqrt(torch.sum(y * y, -1, keepdim=True) / c["d"] + 1e-6)
            y = _to_bf16(_to_bf16(y).to(f64) * weight.to(f64)).to(f64)
        out, h = y.clone(), c["rotary"] // 2
        i = torch.arange(h, device=_DEV)
        first, second = (2 * i, 2 * i + 1) if c["pairs"] == "interleaved" else (i, i + h)
        co, si = st["cos"][positions].to(f64).unsqueeze(1), st["sin"][positions].to(f64).unsqueeze(1)
        out[..., first] = y[..., first] * co - y[..., second] * si
        out[..., second] = y[..., second] * co + y[..., first] * si
        return out

    if c["kind"] == "rope":
        place = torch.cat([torch.arange(int(n), device=_DEV) + int(s) for s, n in zip(st["start"], st["lens_host"])])
        return turned(st["q_in"], place, st["q_norm"]), turned(st["k_in"], place, st["k_norm"])

    def value(pool, side, page, slot):
        s = st["scales"][page, :, slot // c["block"], side].to(f64)
        return pool[page, slot].to(torch.float32).to(f64) * s[..., None], s

    if c["kind"] in ("append", "store"):
        backs = [[], []]
        if c["kind"] == "append":
            # the cache holds what the rotated key is as bf16
            q = turned(st["q_in"], st["lens"].long(), st["q_norm"])
            k = _to_bf16(turned(st["k_new"], st["lens"].long(), st["k_norm"]))
        for b in range(c["B"]):
            begin = int(st["lens_host"][b] if c["kind"] == "append" else st["start"][b])
            end = begin + (1 if c["kind"] == "append" else int(st["lens_host"][b]))
            lo = int(st["offsets"][b])
            p = begin
            while p < end:
                first = p - p % c["block"]
                until = min(first + c["block"], end)
                slot = torch.arange(first % c["ps"], first % c["ps"] + p - first, device=_DEV)
                page = torch.full_like(slot, int(st["table"][b, p // c["ps"]]))
                for side, pool in ((0, st["k"]), (1, st["v"])):
                    if c["kind"] == "append":
                        x = (k, st["v_new"])[side][b:b + 1]
                    else:
                        x = (st["k_in"], st["v_in"])[side][lo + p - begin:lo + until - begin]
                    held = None, None
                    if p > first:
                        old, s = value(pool, side, page, slot)
                        held = old, s[0]
                    y = through(x, held, p - first)
                    # appending reads the whole block back, storing what it stored
                    backs[side].append(y if c["kind"] == "append" else y[p - first:])
                p = until
        empty = torch.zeros(0, c["Hkv"], c["d"], dtype=f64, device=_DEV)
        k_back, v_back = (torch.cat(x) if x else empty for x in backs)
        return (q, k_back, v_back) if c["kind"] == "append" else (k_back, v_back)

    out = torch.zeros(c["B"], c["Hq"], c["d"], dtype=f64, device=_DEV)
    per = c["Hq"] // c["Hkv"]
    for b in range(c["B"]):
        n = int(st["lens_host"][b]) + 1
        t = torch.arange(n, device=_DEV)
        if c["window"] and n > c["window"]:
            t = torch.cat((t[: min(c["sinks"], n - c["window"])], t[n - c["window"]:]))
        page, slot = st["table"][b, t // c["ps"]].long(), t % c["ps"]
        k, v = value(st["k"], 0, page, slot)[0], value(st["v"], 1, page, slot)[0]
        for h in range(c["Hkv"]):
            score = st["q"][b, h * per:(h + 1) * per].to(f64) @ k[:, h].T / math.sqrt(c["d"])
            out[b, h * per:(h + 1) * per] = torch.softmax(score, -1) @ v[:, h]
    return out
