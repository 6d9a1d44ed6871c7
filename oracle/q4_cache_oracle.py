"""CPU oracle for the 4-bit cache, for attention under a window with sinks, and for the page operations.

TEST INFRASTRUCTURE ONLY, like the oracle of the bf16 path: plain numpy in fp64 and Python loops, written from the
definitions, importing nothing of the CUDA path.  bf16 tensors are uint16 bit patterns.
"""
from __future__ import annotations

import numpy as np

from .paged_decode_oracle import bf16_to_f64, f64_to_bf16_rne

NAN = np.uint16(0x7FC0)


def quantise(x_bits, group):
    """bf16 bits [..., d] -> codes uint8 [..., d], scale and minimum bits uint16 [..., d / group].

    m = min x, s = bf16(fp32((max x - m) / 15)), c = clamp(rint((x - m) / s), 0, 15), 0 where s = 0; a group with a
    non-finite element: m = NaN, s = 0, c = 0.  A zero minimum and a zero scale are +0."""
    x = bf16_to_f64(x_bits)
    y = x.reshape(*x.shape[:-1], -1, group)
    bad = ~np.isfinite(y).all(-1)
    y = np.where(bad[..., None], 0.0, y)
    m = y.min(-1) + 0.0
    m = np.where(m == 0, 0.0, m)
    s_bits = f64_to_bf16_rne(((y.max(-1) - m) / 15.0 + 0.0).astype(np.float32).astype(np.float64))    # never -0
    s = bf16_to_f64(s_bits)
    with np.errstate(divide="ignore", invalid="ignore"):
        c = np.where(s[..., None] > 0, np.clip(np.rint((y - m[..., None]) / s[..., None]), 0, 15), 0.0)
    codes = c.astype(np.uint8).reshape(x.shape)
    return codes, np.where(bad, np.uint16(0), s_bits), np.where(bad, NAN, f64_to_bf16_rne(m))


def pack(codes):
    """codes [..., d] -> bytes [..., d / 2], element 2i in the low nibble of byte i."""
    return (codes[..., 0::2] | (codes[..., 1::2] << 4)).astype(np.uint8)


def unpack(packed):
    out = np.empty((*packed.shape[:-1], 2 * packed.shape[-1]), dtype=np.uint8)
    out[..., 0::2], out[..., 1::2] = packed & 15, packed >> 4
    return out


def values(packed, s_bits, m_bits):
    """What packed codes [..., d / 2] under scales and minima [..., G] stand for, fp64 [..., d]; also c * s alone."""
    c = unpack(packed).astype(np.float64)
    g = c.shape[-1] // s_bits.shape[-1]
    cs = c * np.repeat(bf16_to_f64(s_bits), g, axis=-1)
    return cs + np.repeat(bf16_to_f64(m_bits), g, axis=-1), cs


def visible(n, window=0, sinks=0):
    """Positions a row of n tokens attends over."""
    t = np.arange(max(n, 0))
    return t if not window else t[(t < sinks) | (t >= n - window)]


def attention(q_bits, fetch, lens, Hkv, window=0, sinks=0, scale=None, slack=False):
    """softmax(scale q K^T) V over each row's visible positions, fp64 [B, Hq, d].

    ``fetch(b, h, positions)`` -> (K, V, |V| weights) fp64 [n, d]; lens[b] = tokens of row b (<= 0: output 0).  With
    ``slack`` also returns sum_t p_t w_t of the third item, the scale of the weights' rounding errors."""
    B, Hq, d = q_bits.shape
    scale = 1.0 / np.sqrt(d) if scale is None else scale
    out, room = np.zeros((B, Hq, d)), np.zeros((B, Hq, d))
    per = Hq // Hkv
    q = bf16_to_f64(q_bits)
    for b in range(B):
        t = visible(int(lens[b]), window, sinks)
        if t.size == 0:
            continue
        for h in range(Hkv):
            K, V, W = fetch(b, h, t)
            s = (q[b, h * per:(h + 1) * per] @ K.T) * scale
            p = np.exp(s - s.max(-1, keepdims=True))
            p /= p.sum(-1, keepdims=True)
            out[b, h * per:(h + 1) * per] = p @ V
            room[b, h * per:(h + 1) * per] = p @ W
    return (out, room) if slack else out


# ---- pages ---------------------------------------------------------------------------------------------------


class Pages:
    """Block table, lengths and reference counts as plain Python; pools as numpy arrays [num_pages, slots, bytes...]
    or, with segments, [num_pages, segments, slots, ...] (``slot_axis`` per pool)."""

    def __init__(self, table, lens, refs, page_size, pools=()):
        self.table, self.lens, self.refs = table.copy(), lens.copy(), refs.copy()
        self.ps, self.pools = page_size, [(p.copy(), axis) for p, axis in pools]

    def pages(self, n):
        return -(-int(n) // self.ps)

    def _free(self):
        return [int(p) for p in np.nonzero(self.refs == 0)[0]]

    def reserve(self, new_tokens):
        free, exhausted = self._free(), False
        for r in range(len(self.lens)):
            n = int(self.lens[r])
            if n < 0:
                continue
            first, last = self.pages(n), self.pages(n + new_tokens)
            if last > self.table.shape[1] or last == first:
                continue
            if exhausted or last - first > len(free):
                exhausted = True
                continue
            for i in range(first, last):
                page = free.pop(0)
                self.table[r, i], self.refs[page] = page, 1

    def fork(self, pairs):
        free = self._free()
        lens = self.lens.copy()
        for parent, child in pairs:
            n = int(lens[parent])
            self.lens[child] = -1
            if n < 0 or self.pages(n) > self.table.shape[1]:
                continue
            full, part = divmod(n, self.ps)
            if part and not free:
                continue
            for i in range(full):
                self.table[child, i] = self.table[parent, i]
                self.refs[self.table[parent, i]] += 1
            if part:
                page = free.pop(0)
                self.refs[page] = 1
                self.table[child, full] = page
                for pool, axis in self.pools:
                    at = (slice(None),) * (axis - 1) + (slice(0, part),)
                    pool[page][at] = pool[self.table[parent, full]][at]
            self.lens[child] = n

    def release(self, rows):
        for r in rows:
            n = int(self.lens[r])
            for i in range(self.pages(max(n, 0))):
                self.refs[self.table[r, i]] -= 1
            self.lens[r] = -1

    def compact(self):
        live = int((self.refs > 0).sum())
        to = [int(p) for p in np.nonzero(self.refs[:live] == 0)[0]]
        old = [live + int(p) for p in np.nonzero(self.refs[live:] > 0)[0]]
        place = dict(zip(old, to))
        for r in range(len(self.lens)):
            for i in range(self.pages(max(int(self.lens[r]), 0))):
                self.table[r, i] = place.get(int(self.table[r, i]), self.table[r, i])
        for a, b in zip(old, to):
            self.refs[b], self.refs[a] = self.refs[a], 0
            for pool, _ in self.pools:
                pool[b] = pool[a]
        return live
