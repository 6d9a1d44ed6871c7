"""CPU oracle for the 8-bit cache and the scaled rotary tables.

TEST INFRASTRUCTURE ONLY, like the other oracles: plain numpy in fp64 (the tables in extended precision) and Python loops,
written from the definitions, importing nothing of the CUDA path.  bf16 tensors are uint16 bit patterns, codes uint8.
"""
from __future__ import annotations

import numpy as np

from .paged_decode_oracle import bf16_to_f64

INT8, E4M3 = "int8", "e4m3"
LARGEST = {INT8: 127.0, E4M3: 448.0}
TOP = {INT8: 121, E4M3: 119}


def _e4m3_values():
    """What the 256 bit patterns stand for."""
    b = np.arange(256)
    e, m = (b >> 3) & 15, b & 7
    v = np.where(e == 0, m * 2.0**-9, (8 + m) * 2.0 ** (e - 10.0))
    v[(b & 0x7F) == 0x7F] = np.nan
    return np.where(b & 0x80, -v, v)


E4M3_VALUES = _e4m3_values()


def code_values(codes, fmt):
    """uint8 codes -> what they stand for under the scale 1, fp64."""
    return codes.view(np.int8).astype(np.float64) if fmt == INT8 else E4M3_VALUES[codes]


def encode(y, fmt):
    """fp64 values (already divided by the scale) -> uint8 codes: nearest, ties to even, clamped; NaN -> anything."""
    y = np.clip(np.where(np.isnan(y), 0.0, y), -LARGEST[fmt], LARGEST[fmt])
    if fmt == INT8:
        return np.rint(y).astype(np.int8).view(np.uint8)
    a = np.abs(y)
    _, e = np.frexp(a)                                     # a in [2^(e-1), 2^e): steps of 2^(e-4), 2^-9 at the bottom
    step = np.ldexp(1.0, np.maximum(e - 4, -9))
    a = np.rint(a / step) * step                           # an even count of steps is an even fraction
    code = np.searchsorted(E4M3_VALUES[:127], a).astype(np.uint8)
    return code | np.where(np.signbit(y), 0x80, 0).astype(np.uint8)


def needed(x, fmt):
    """The scale that values x [..., d] of one block and head need: least 2^e with max |x| <= M 2^e; NaN if one is not finite."""
    if not np.isfinite(x).all():
        return np.nan
    e = -100
    most = float(np.abs(x).max()) if x.size else 0.0
    while e < TOP[fmt] and most > LARGEST[fmt] * 2.0**e:
        e += 1
    return 2.0**e


def write(codes, scales, x_bits, before, fmt):
    """Writes x_bits [n, d] behind `before` tokens of a block: codes uint8 [block, d] is changed in place, the new scale returned."""
    x = bf16_to_f64(x_bits)
    s = needed(x, fmt)
    if before:
        if np.isnan(scales) or np.isnan(s):
            s = np.nan
        elif s > scales:
            codes[:before] = encode(code_values(codes[:before], fmt) * (float(scales) / s), fmt)
        else:
            s = float(scales)
    codes[before:before + len(x)] = encode(x / s, fmt)
    return s


class Cache:
    """Codes uint8 [page, slot, head, d] of K and V and scales [page, head, block, side], changed as the library's calls do."""

    def __init__(self, k, v, scales, fmt):
        self.pools, self.scales, self.fmt = (k, v), scales, fmt
        self.ps, self.block = k.shape[1], k.shape[1] // scales.shape[2]

    def store(self, x, side, table_row, start):
        """Tokens x [n, heads, d] (bf16 bits) at positions start, start + 1, ... of one row."""
        at, n = 0, len(x)
        while at < n:
            p = start + at
            page, slot = table_row[p // self.ps], p % self.ps
            blk, before = slot // self.block, slot % self.block
            m = min(self.block - before, n - at)
            for h in range(x.shape[1]):
                codes = self.pools[side][page, blk * self.block:(blk + 1) * self.block, h].copy()
                self.scales[page, h, blk, side] = write(codes, self.scales[page, h, blk, side], x[at:at + m, h], before, self.fmt)
                self.pools[side][page, blk * self.block:blk * self.block + before + m, h] = codes[:before + m]
            at += m

    def read(self, side, table_row, positions, h=slice(None)):
        """fp64 values [n, (heads,) d]; NaN where the scale is."""
        page, slot = table_row[positions // self.ps], positions % self.ps
        c = code_values(self.pools[side][page, slot], self.fmt)
        s = self.scales[page, :, slot // self.block, side].astype(np.float64)
        return (c * s[..., None])[:, h]


def frequencies(rotary_dim, base, scaling="none", factor=1.0, original=0.0, low=0.0, high=0.0):
    """f_i in extended precision."""
    L = np.longdouble
    b = L(base)
    if scaling == "base":
        b = b * L(factor) ** (L(rotary_dim) / L(rotary_dim - 2))
    f = b ** (-2 * np.arange(rotary_dim // 2, dtype=L) / L(rotary_dim))
    if scaling == "linear":
        f = f / L(factor)
    if scaling == "ramp":
        pi = L("3.14159265358979323846264338327950288")
        g = np.clip((L(original) * f / (2 * pi) - L(low)) / (L(high) - L(low)), 0, 1)
        f = g * f + (1 - g) * f / L(factor)
    return f


def tables(first, positions, f, magnitude=1.0):
    """Cosines and sines [positions, R/2], extended precision."""
    ang = np.arange(first, first + positions, dtype=np.longdouble)[:, None] * f[None, :]
    return np.longdouble(magnitude) * np.cos(ang), np.longdouble(magnitude) * np.sin(ang)
