"""What is measured of the 4-bit paged cache, the attention with sinks and the page operations.

Every case is a plain dict; ``run`` makes one pass through an operator, either in its plain form (elementary torch
operations in 32 or 64 bits) or, with ``own`` set, by the calls a serving program makes.

Kinds of cases
  append   RoPE of the new q and k, the new k and v quantised into their 4-bit pages, and the written token read back
  store    a batch of prompts quantised into the 4-bit pages and read back (a prefix that is used again)
  attn     decode attention over the 4-bit cache, optionally with a window and sinks
  sinks    decode attention over the bf16 cache with a sliding window whose first tokens stay visible
  fork     sequences forked from parents (full pages shared, the partly filled page copied), then released again
  compact  live pages moved to the lowest page ids, tables and reference counts rewritten

The 4-bit format: a group of ``group`` consecutive elements of one (token, head) holds m = min x and
s = bf16((max x - min x) / 15) as bf16 and codes c = rint((x - m) / s); it stands for c * s + m.  Element 2i is the low
nibble of byte i.  Parameters are [page, head, slot, K or V, group, (s, m)].
"""
import math

import numpy as np
import torch

own = False

_DEV = "cuda"


def listed():
    return [
        # one token of each of 8 requests, the middle bucket of the graph sweep: latency of a short step
        dict(name="append_b8", kind="append", B=8, Hq=28, Hkv=4, d=128, ps=32, group=64, lo=512, hi=2048, len_seed=51),
        # the largest bucket of the same sweep
        dict(name="append_b256", kind="append", B=256, Hq=28, Hkv=4, d=128, ps=32, group=64, lo=512, hi=2048, len_seed=54),
        # 32 prompts of up to 4096 tokens entering the cache together and read back for a prefix
        dict(name="store_b32", kind="store", B=32, Hq=32, Hkv=8, d=128, ps=16, group=64, lo=17, hi=4096, len_seed=7),
        # the smallest decode step: 512 tokens, two KV heads of 64 elements
        dict(name="attn_tiny", kind="attn", B=1, Hq=8, Hkv=2, d=64, ps=16, group=32, lo=512, hi=512, len_seed=1, window=0, sinks=0),
        # continuous batching: 64 requests of 128 to 8192 tokens
        dict(name="attn_b64", kind="attn", B=64, Hq=32, Hkv=8, d=128, ps=16, group=64, lo=128, hi=8192, len_seed=3, window=0, sinks=0),
        # long contexts, eight query heads per KV head
        dict(name="attn_long", kind="attn", B=4, Hq=64, Hkv=8, d=128, ps=16, group=64, lo=131071, hi=131071, len_seed=4, window=0, sinks=0),
        # one long conversation held to a window of 1024 tokens and four sinks
        dict(name="sinks_b1", kind="sinks", B=1, Hq=32, Hkv=8, d=128, ps=16, lo=20000, hi=20000, len_seed=5, window=1024, sinks=4),
        # a batch under the 4096-token window, some rows still shorter than it
        dict(name="sinks_b32", kind="sinks", B=32, Hq=32, Hkv=8, d=128, ps=16, lo=2048, hi=12288, len_seed=6, window=4096, sinks=100),
        # eight beams of one request, one layer's pools
        dict(name="fork_b8", kind="fork", pools=2, pages=1024, ps=16, heads=8, d=128, parents=1, forks=8, lo=1001, hi=1001, len_seed=8),
        # 128 forks of 64 requests, sixteen layers that share one block table
        dict(name="fork_b128", kind="fork", pools=32, pages=2560, ps=16, heads=8, d=128, parents=64, forks=128, lo=100, hi=600, len_seed=9),
        # a small pool after a few requests ended
        dict(name="compact_small", kind="compact", pools=2, pages=512, ps=16, heads=2, d=64, rows=4, lo=300, hi=900, len_seed=10),
        # the 40000-page pool of the continuous batch, two fifths of it live and scattered
        dict(name="compact_40k", kind="compact", pools=2, pages=40000, ps=16, heads=8, d=128, rows=64, lo=128, hi=8000, len_seed=11),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["append", "store", "attn", "attn", "sinks", "fork", "compact"])
    c = dict(kind=kind, len_seed=rng.randrange(1 << 20))
    d, hkv = rng.choice([64, 128, 128]), rng.choice([1, 2, 3, 4, 8])
    c.update(d=d, ps=rng.choice([16, 32, 48, 64, 128]))
    if kind in ("append", "store", "attn", "sinks"):
        c.update(Hkv=hkv, Hq=hkv * rng.choice([1, 2, 3, 4, 7, 8, 16]))
        if kind != "sinks":
            c.update(group=rng.choice([g for g in (32, 64, 128) if g <= d]))
    if kind == "append":
        c.update(B=_log(rng, 1, 256), lo=rng.choice([0, 1, 100]), hi=_log(rng, 128, 4096))
    elif kind == "store":
        c.update(B=_log(rng, 1, 32), lo=rng.choice([0, 1, 17]), hi=_log(rng, 32, 4096))
    elif kind in ("attn", "sinks"):
        c.update(B=_log(rng, 1, 64))
        hi = _log(rng, 16, max(64, 262144 // c["B"]))
        w = rng.randrange(1, hi + 1)
        window = w if kind == "sinks" or rng.random() < 0.4 else 0
        c.update(lo=rng.choice([0, 1, max(1, hi // 2)]), hi=hi, window=window, sinks=_log(rng, 1, 600) if window else 0)
    elif kind == "fork":
        c.update(pools=rng.choice([1, 2, 4, 16]), heads=hkv, parents=_log(rng, 1, 32), forks=_log(rng, 1, 128), lo=rng.choice([0, 1, 33]), hi=_log(rng, 64, 500))
        c["pages"] = c["parents"] * (c["hi"] // c["ps"] + 1) + c["forks"] + _log(rng, 4, 500)
    else:
        c.update(pools=rng.choice([1, 2]), heads=hkv, rows=_log(rng, 1, 40), lo=rng.choice([0, 1, 33]), hi=_log(rng, 64, 4000))
        c["pages"] = c["rows"] * (c["hi"] // c["ps"] + 2) + _log(rng, 4, 4000)
    return c


def _lengths(c, n):
    return np.random.default_rng(c["len_seed"]).integers(c["lo"], c["hi"] + 1, size=n).astype(np.int64)


def _visible(c, n):
    """Tokens a row of n tokens attends over."""
    w, s = c["window"], c["sinks"]
    return n if w == 0 else np.minimum(n, w) + np.minimum(s, np.maximum(n - w, 0))


def work(c):
    k = c["kind"]
    if k in ("fork", "compact"):
        page = c["ps"] * c["heads"] * c["d"] * 2 * c["pools"]
    if k == "fork":
        n = _lengths(c, c["parents"])[np.arange(c["forks"]) % c["parents"]]
        moved = int((n % c["ps"]).sum()) * (page // c["ps"])
        return {"bytes": 2 * moved + int((n // c["ps"] + 1).sum()) * 16, "flops": 0}
    if k == "compact":
        n = _lengths(c, c["rows"])
        live = int((-(-n // c["ps"])).sum())
        return {"bytes": 2 * page * int(round(live * (1 - live / c["pages"]))) + 8 * c["pages"] + 8 * live, "flops": 0}
    kv = c["Hkv"] * c["d"]
    if k == "append":
        B = c["B"]
        q4 = 2 * c["Hkv"] * (c["d"] // 2 + 4 * (c["d"] // c["group"]))
        return {"bytes": B * (4 * c["Hq"] * c["d"] + 4 * kv + 2 * q4 + 4 * kv + 4 * c["d"]), "flops": B * 6 * (c["Hq"] + 2 * c["Hkv"]) * c["d"]}
    if k == "store":
        q4 = 2 * c["Hkv"] * (c["d"] // 2 + 4 * (c["d"] // c["group"]))
        t = int(_lengths(c, c["B"]).sum())
        return {"bytes": t * (8 * kv + 2 * q4) + 4, "flops": t * 8 * kv}
    t = int(_visible(c, _lengths(c, c["B"]) + 1).sum())
    token = 4 * kv if k == "sinks" else 2 * c["Hkv"] * (c["d"] // 2 + 4 * (c["d"] // c["group"]))
    return {"bytes": t * token + 4 * c["B"] * c["Hq"] * c["d"], "flops": 4 * t * c["Hq"] * c["d"]}


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


def _rope(c, positions):
    i = np.arange(c["d"] // 2, dtype=np.float64)
    ang = np.arange(positions, dtype=np.float64)[:, None] * np.power(500000.0, -2.0 * i / c["d"])[None, :]
    return torch.from_numpy(np.cos(ang).astype(np.float32)).to(_DEV), torch.from_numpy(np.sin(ang).astype(np.float32)).to(_DEV)


def _q4_pools(gen, c, num_pages, used):
    """Codes and parameters of a cache whose values have unit variance; what no row refers to reads as NaN."""
    shape = (num_pages, c["ps"], c["Hkv"], c["d"] // 2)
    k = torch.randint(0, 256, shape, generator=gen, device=_DEV, dtype=torch.uint8)
    v = torch.randint(0, 256, shape, generator=gen, device=_DEV, dtype=torch.uint8)
    p = torch.full((num_pages, c["Hkv"], c["ps"], 2, c["d"] // c["group"], 2), float("nan"), device=_DEV, dtype=torch.bfloat16)
    s = 0.2 + 0.05 * torch.rand(len(used), *p.shape[1:5], generator=gen, device=_DEV)
    p[used, ..., 0] = s.to(torch.bfloat16)
    p[used, ..., 1] = (-7.5 * s + 0.1 * torch.randn(s.shape, generator=gen, device=_DEV)).to(torch.bfloat16)
    return k, v, p


def prepare(case, seed):
    c = case
    gen = torch.Generator(device=_DEV).manual_seed(seed)
    st = {"case": c}
    if c["kind"] in ("append", "store", "attn", "sinks"):
        lens = _lengths(c, c["B"])
        room = 0 if c["kind"] == "store" else 1
        need = -(-(lens + room) // c["ps"])
        num_pages = int(need.sum() * 1.25) + 2
        st["table"], used = _table(gen, need, num_pages, max(1, int(need.max())))
        st["lens_host"] = lens
        st["lens"] = torch.from_numpy(lens.astype(np.int32)).to(_DEV)
        st["num_pages"] = num_pages
    if c["kind"] == "append":
        st["k"], st["v"], st["p"] = _q4_pools(gen, c, num_pages, used)
        st["q_in"], st["k_new"], st["v_new"] = (_normal(gen, c["B"], h, c["d"]) for h in (c["Hq"], c["Hkv"], c["Hkv"]))
        st["q_out"], st["k_back"], st["v_back"] = torch.zeros_like(st["q_in"]), torch.zeros_like(st["k_new"]), torch.zeros_like(st["v_new"])
        st["cos"], st["sin"] = _rope(c, int(lens.max()) + 1)
        st["offsets"] = torch.arange(c["B"] + 1, device=_DEV, dtype=torch.int32)
    elif c["kind"] == "store":
        st["k"], st["v"], st["p"] = _q4_pools(gen, c, num_pages, used)
        total = int(lens.sum())
        st["k_in"], st["v_in"] = (_normal(gen, total, c["Hkv"], c["d"]) for _ in range(2))
        st["k_back"], st["v_back"] = torch.zeros_like(st["k_in"]), torch.zeros_like(st["v_in"])
        st["start"] = torch.zeros(c["B"], device=_DEV, dtype=torch.int32)
        st["offsets"] = torch.from_numpy(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)).to(_DEV)
    elif c["kind"] == "attn":
        st["k"], st["v"], st["p"] = _q4_pools(gen, c, num_pages, used)
        # slots behind a row's last token hold anything
        last, slot = torch.from_numpy(lens // c["ps"]).to(_DEV), torch.from_numpy(lens % c["ps"]).to(_DEV)
        page = st["table"][torch.arange(c["B"], device=_DEV), last].long()
        behind = torch.arange(c["ps"], device=_DEV)[None, :] > slot[:, None]
        tail = st["p"][page]
        tail[behind[:, None, :].expand(-1, c["Hkv"], -1)] = float("nan")
        st["p"][page] = tail
        st["q"] = _normal(gen, c["B"], c["Hq"], c["d"])
        st["out"] = torch.zeros_like(st["q"])
    elif c["kind"] == "sinks":
        st["k"] = _normal(gen, num_pages, c["ps"], c["Hkv"], c["d"])
        st["v"] = _normal(gen, num_pages, c["ps"], c["Hkv"], c["d"])
        spare = torch.ones(num_pages, dtype=torch.bool, device=_DEV)
        spare[used] = False
        st["k"][spare] = float("nan")
        st["v"][spare] = float("nan")
        st["q"] = _normal(gen, c["B"], c["Hq"], c["d"])
        st["out"] = torch.zeros_like(st["q"])
    elif c["kind"] == "fork":
        rows = c["parents"] + c["forks"]
        lens = np.full(rows, -1, dtype=np.int64)
        lens[: c["parents"]] = _lengths(c, c["parents"])
        need = -(-np.maximum(lens, 0) // c["ps"])
        st["table"], used = _table(gen, need, c["pages"], max(1, int(need.max()) + 1))
        st["lens"] = torch.from_numpy(lens.astype(np.int32)).to(_DEV)
        st["refs"] = torch.zeros(c["pages"], dtype=torch.int32, device=_DEV)
        st["refs"][used] = 1
        i = np.arange(c["forks"])
        st["pairs"] = torch.from_numpy(np.stack([i % c["parents"], c["parents"] + i], 1).astype(np.int32)).to(_DEV)
        st["children"] = st["pairs"][:, 1].contiguous()
        st["pools"] = torch.randint(-32768, 32767, (c["pools"], c["pages"], c["ps"], c["heads"], c["d"]), generator=gen, device=_DEV, dtype=torch.int16)
    else:
        lens = _lengths(c, c["rows"])
        need = -(-lens // c["ps"])
        st["table"], used = _table(gen, need, c["pages"], max(1, int(need.max())))
        st["lens"] = torch.from_numpy(lens.astype(np.int32)).to(_DEV)
        st["refs"] = torch.zeros(c["pages"], dtype=torch.int32, device=_DEV)
        st["refs"][used] = 1
        st["pools"] = torch.randint(-32768, 32767, (c["pools"], c["pages"], c["ps"], c["heads"], c["d"]), generator=gen, device=_DEV, dtype=torch.int16)
        # the tables of the next step: the present ones stay as they are for the step still in flight
        st["table_out"], st["refs_out"] = torch.zeros_like(st["table"]), torch.zeros_like(st["refs"])
        st["live"] = torch.zeros(1, dtype=torch.int32, device=_DEV)
    return st


# ---- the plain forms --------------------------------------------------------------------------------------------


def _to_bf16(x):
    """Nearest-even bf16 of 64-bit values, rounded once."""
    m, e = torch.frexp(x)
    return torch.ldexp(torch.round(m * 256.0), e - 8).to(torch.bfloat16)


def _quantise(x, group):
    """bf16 [..., d] -> codes [..., d], scale and minimum [..., d / group]."""
    y = x.double().unflatten(-1, (-1, group))
    m = y.amin(-1)
    s = ((y.amax(-1) - m) / 15.0).float().to(torch.bfloat16)
    step = s.double()[..., None]
    c = torch.where(step > 0, torch.round((y - m[..., None]) / torch.where(step > 0, step, 1.0)).clamp(0, 15), 0.0)
    return c.flatten(-2).to(torch.uint8), s, m.to(torch.bfloat16)


def _values(codes, s, m):
    """Packed codes [..., d / 2] with scale and minimum [..., G] -> the 32-bit values they stand for."""
    c = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).float()
    return (c.unflatten(-1, (s.shape[-1], -1)) * s.float()[..., None] + m.float()[..., None]).flatten(-2)


def _write(st, page, slot, x, side, pool):
    c, s, m = _quantise(x, st["case"]["group"])
    pool[page, slot] = c[..., 0::2] | (c[..., 1::2] << 4)
    st["p"][page, :, slot, side] = torch.stack((s, m), -1)


def _read(st, page, slot, side, pool):
    p = st["p"][page, :, slot, side]
    return _values(pool[page, slot], p[..., 0], p[..., 1]).to(torch.bfloat16)


def _rotate(x, cos, sin):
    a, b = x.double().chunk(2, -1)
    return _to_bf16(torch.cat((a * cos - b * sin, b * cos + a * sin), -1))


def _plain_append(st):
    c, pos = st["case"], st["lens"].long()
    cos, sin = st["cos"][pos].double()[:, None], st["sin"][pos].double()[:, None]
    page = st["table"].gather(1, (pos // c["ps"])[:, None])[:, 0].long()
    st["q_out"].copy_(_rotate(st["q_in"], cos, sin))
    _write(st, page, pos % c["ps"], _rotate(st["k_new"], cos, sin), 0, st["k"])
    _write(st, page, pos % c["ps"], st["v_new"], 1, st["v"])
    st["k_back"].copy_(_read(st, page, pos % c["ps"], 0, st["k"]))
    st["v_back"].copy_(_read(st, page, pos % c["ps"], 1, st["v"]))
    return st["q_out"], st["k_back"], st["v_back"]


def _plain_store(st):
    c, off = st["case"], st["offsets"].long()
    t = torch.arange(st["k_in"].shape[0], device=_DEV)
    row = torch.searchsorted(off, t, right=True) - 1
    pos = t - off[row] + st["start"].long()[row]
    page, slot = st["table"][row, pos // c["ps"]].long(), pos % c["ps"]
    _write(st, page, slot, st["k_in"], 0, st["k"])
    _write(st, page, slot, st["v_in"], 1, st["v"])
    st["k_back"].copy_(_read(st, page, slot, 0, st["k"]))
    st["v_back"].copy_(_read(st, page, slot, 1, st["v"]))
    return st["k_back"], st["v_back"]


def _plain_attention(st):
    c = st["case"]
    n = st["lens"].long() + 1
    page = st["table"].long()
    if c["kind"] == "attn":
        p = st["p"][page].transpose(2, 3)                                  # [B, pages, slot, head, side, group, 2]
        k = _values(st["k"][page], p[..., 0, :, 0], p[..., 0, :, 1]).flatten(1, 2)
        v = _values(st["v"][page], p[..., 1, :, 0], p[..., 1, :, 1]).flatten(1, 2)
    else:
        k, v = st["k"][page].float().flatten(1, 2), st["v"][page].float().flatten(1, 2)
    t = torch.arange(k.shape[1], device=_DEV)[None, :]
    seen = t < n[:, None]
    if c["window"]:
        seen = seen & ((t >= (n - c["window"])[:, None]) | (t < c["sinks"]))
    q = st["q"].float().unflatten(1, (c["Hkv"], -1))
    k = torch.where(seen[:, :, None, None], k, 0.0)
    v = torch.where(seen[:, :, None, None], v, 0.0)
    s = torch.einsum("bhgd,bthd->bhgt", q, k) / math.sqrt(c["d"])
    s = torch.where(seen[:, None, None, :], s, float("-inf"))
    e = torch.exp(s - s.amax(-1, keepdim=True))
    o = torch.einsum("bhgt,bthd->bhgd", e / e.sum(-1, keepdim=True), v)
    st["out"].copy_(o.flatten(1, 2))
    return st["out"]


def _plain_fork(st):
    c = st["case"]
    table, lens, refs = st["table"], st["lens"], st["refs"]
    parent, child = st["pairs"][:, 0].long(), st["pairs"][:, 1].long()
    n = lens[parent].long()
    full, part = n // c["ps"], n % c["ps"]
    at = torch.arange(table.shape[1], device=_DEV)[None, :]
    shared = at < full[:, None]
    table[child] = torch.where(shared, table[parent], table[child])
    refs.index_add_(0, table[child][shared].long(), torch.ones_like(table[child][shared]))
    grows = torch.nonzero(part > 0)[:, 0]
    fresh = torch.nonzero(refs == 0)[: len(grows), 0]
    old = table[parent[grows], full[grows]].long()
    table[child[grows], full[grows]] = fresh.to(torch.int32)
    refs[fresh] = 1
    lens[child] = n.to(torch.int32)
    keep = (torch.arange(c["ps"], device=_DEV)[None, :] < part[grows][:, None])[:, :, None, None]
    pool = st["pools"]
    pool[:, fresh] = torch.where(keep, pool[:, old], pool[:, fresh])
    # the forks are dropped again
    held = at < (-(-n // c["ps"]))[:, None]
    gone = table[child][held].long()
    refs.index_add_(0, gone, torch.full_like(gone, -1, dtype=torch.int32))
    lens[child] = -1
    return table, lens, refs, pool


def _plain_compact(st):
    c, refs = st["case"], st["refs"]
    ids = torch.arange(c["pages"], device=_DEV)
    live = int((refs > 0).sum())
    to = torch.nonzero((refs == 0) & (ids < live))[:, 0]
    old = torch.nonzero((refs > 0) & (ids >= live))[:, 0]
    place = ids.clone()
    place[old] = to
    n = st["lens"].long().clamp(min=0)
    held = torch.arange(st["table"].shape[1], device=_DEV)[None, :] < (-(-n // c["ps"]))[:, None]
    st["table_out"].copy_(torch.where(held, place[st["table"].long()].to(torch.int32), st["table"]))
    st["refs_out"].copy_(refs)
    st["refs_out"][to] = refs[old]
    st["refs_out"][old] = 0
    st["live"].fill_(live)
    st["pools"][:, to] = st["pools"][:, old]
    return st["table_out"], st["refs_out"], st["live"], st["pools"]


# ---- the framework's calls --------------------------------------------------------------------------------------


def _handle(st):
    """What a serving program keeps from step to step: the plan, the workspace and the objects that hold its buffers."""
    from paper_2606_07665_b200 import runner

    c = st["case"]
    if c["kind"] in ("append", "store", "attn"):
        cache = runner.Q4Cache(st["k"], st["v"], st["p"], page_size=c["ps"])
        if c["kind"] == "store":
            return cache
        return runner.Q4DecodeStep(cache, st["table"], st["lens"], Hq=c["Hq"], lens_host=st["lens_host"], window=c.get("window", 0), sinks=c.get("sinks", 0), rope_cos=st.get("cos"), rope_sin=st.get("sin"))
    if c["kind"] == "sinks":
        return runner.PagedAttention(st["k"], st["v"], st["table"], st["lens"], Hq=c["Hq"], lens_host=st["lens_host"], window=c["window"], sinks=c["sinks"])
    return runner.CachePages(list(st["pools"]), st["table"], st["lens"], st["refs"], page_size=c["ps"])


def _own(st):
    kind = st["case"]["kind"]
    if "handle" not in st:
        st["handle"] = _handle(st)
    h = st["handle"]
    if kind == "append":
        h.append(st["q_in"], st["k_new"], st["v_new"], q_out=st["q_out"])
        h.cache.load(st["table"], st["lens"], st["offsets"], k_out=st["k_back"], v_out=st["v_back"])
        return st["q_out"], st["k_back"], st["v_back"]
    if kind == "store":
        h.store(st["k_in"], st["v_in"], st["table"], st["start"], st["offsets"])
        h.load(st["table"], st["start"], st["offsets"], k_out=st["k_back"], v_out=st["v_back"])
        return st["k_back"], st["v_back"]
    if kind in ("attn", "sinks"):
        h.attention(st["q"], out=st["out"])
        return st["out"]
    if kind == "fork":
        h.fork(st["pairs"])
        h.release(st["children"])
        return st["table"], st["lens"], st["refs"], st["pools"]
    h.compact(table_out=st["table_out"], refs_out=st["refs_out"], live_out=st["live"])
    return st["table_out"], st["refs_out"], st["live"], st["pools"]


def run(state):
    if own:
        return _own(state)
    kind = state["case"]["kind"]
    plain = {"append": _plain_append, "store": _plain_store, "attn": _plain_attention, "sinks": _plain_attention, "fork": _plain_fork, "compact": _plain_compact}
    return plain[kind](state)


# ---- 64 bits, from the definitions ------------------------------------------------------------------------------


def exact(case, seed):
    c = case
    if c["kind"] in ("fork", "compact"):
        return None                                                        # whole numbers only
    st = prepare(case, seed)
    f64 = torch.float64

    def through_format(x):
        """What [n, heads, d] values read back as."""
        out = torch.empty(x.shape, dtype=f64, device=_DEV)
        for g in range(0, c["d"], c["group"]):
            part = x[..., g:g + c["group"]].to(f64)
            lo, hi = part.min(-1, keepdim=True).values, part.max(-1, keepdim=True).values
            s = ((hi - lo) / 15).to(torch.float32).to(torch.bfloat16).to(f64)
            code = torch.where(s == 0, torch.zeros_like(part), torch.clamp(torch.round((part - lo) / s), 0, 15))
            out[..., g:g + c["group"]] = code * s + lo
        return out

    if c["kind"] == "store":
        return through_format(st["k_in"]), through_format(st["v_in"])
    if c["kind"] == "append":
        half = c["d"] // 2

        def turned(x):
            y = torch.empty(x.shape, dtype=f64, device=_DEV)
            for b in range(c["B"]):
                co, si = st["cos"][int(st["lens_host"][b])].to(f64), st["sin"][int(st["lens_host"][b])].to(f64)
                y[b, :, :half] = x[b, :, :half].to(f64) * co - x[b, :, half:].to(f64) * si
                y[b, :, half:] = x[b, :, half:].to(f64) * co + x[b, :, :half].to(f64) * si
            return y

        # the cache holds what the rotated key is as bf16
        return turned(st["q_in"]), through_format(_to_bf16(turned(st["k_new"]))), through_format(st["v_new"])
    out = torch.zeros(c["B"], c["Hq"], c["d"], dtype=f64, device=_DEV)
    per = c["Hq"] // c["Hkv"]
    for b in range(c["B"]):
        n = int(st["lens_host"][b]) + 1
        t = torch.arange(n, device=_DEV)
        if c["window"] and n > c["window"]:
            t = torch.cat((t[: min(c["sinks"], n - c["window"])], t[n - c["window"]:]))
        page, slot = st["table"][b, t // c["ps"]].long(), t % c["ps"]
        for h in range(c["Hkv"]):
            kv = []
            for side, pool in ((0, st["k"]), (1, st["v"])):
                x = pool[page, slot, h]
                if c["kind"] == "attn":
                    p = st["p"][page, h, slot, side].to(f64)
                    y = torch.empty(len(t), c["d"], dtype=f64, device=_DEV)
                    y[:, 0::2], y[:, 1::2] = (x & 15).to(f64), (x >> 4).to(f64)
                    x = y * p[..., 0].repeat_interleave(c["group"], -1) + p[..., 1].repeat_interleave(c["group"], -1)
                kv.append(x.to(f64))
            score = st["q"][b, h * per:(h + 1) * per].to(f64) @ kv[0].T / math.sqrt(c["d"])
            out[b, h * per:(h + 1) * per] = torch.softmax(score, -1) @ kv[1]
    return out
