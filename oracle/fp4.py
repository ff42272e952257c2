"""fp64 oracle of the 4-bit cache: e2m1 codes with one power-of-two scale for 32 dims of a token, and
the stored tiles.

TEST INFRASTRUCTURE ONLY (see kvprm_oracle). Token-major caches are codes [pages][kv-heads][16][d] and
scale bytes [pages][kv-heads][16][d / 32]; ``store`` / ``load`` turn them into the pools' bytes and back, a
byte at a time by the formulas of the C header.
"""
from __future__ import annotations

import numpy as np

PAGE, GROUP = 16, 32
VALUES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def encode(x: np.ndarray):
    """float values [..., d] -> codes [..., d], scale bytes [..., d / 32]."""
    g = np.asarray(x, dtype=np.float64).reshape(*x.shape[:-1], -1, GROUP)
    bad = ~np.all(np.isfinite(g), axis=-1)
    a = np.where(bad[..., None], 0.0, np.abs(g))
    top = a.max(axis=-1)
    k = np.full(top.shape, -100)
    for e in range(-100, 125):  # the smallest exponent that is enough
        k = np.where(7 * 2.0 ** e < top, e + 1, k)
    y = a / 2.0 ** k[..., None]
    dist = np.abs(y[..., None] - VALUES)
    near = dist.min(axis=-1, keepdims=True)
    even = np.array([0, 1] * 4)
    code = np.argmin(np.where(dist == near, even, 2), axis=-1)  # of two as near, the even one
    code = np.where(bad[..., None], 0, code | np.where(np.signbit(g), 8, 0))
    return code.reshape(x.shape).astype(np.uint8), np.where(bad, 255, k + 127).astype(np.uint8)


def decode(code: np.ndarray, scale: np.ndarray) -> np.ndarray:
    v = np.where(code >> 3 != 0, -1.0, 1.0) * VALUES[code & 7]
    s = np.where(scale == 255, np.nan, 2.0 ** (scale.astype(np.float64) - 127))
    return v * np.repeat(s, GROUP, axis=-1)


def places(d: int, part: int):
    """Byte and nibble of every (slot, dim)'s code in a tile, and the byte of its scale."""
    s, m = np.meshgrid(np.arange(PAGE), np.arange(d), indexing="ij")
    if part == 0:
        return ((m // 32) * 16 + s) * 16 + m % 32 // 2, m % 2, 8 * d + (m // 32) * 16 + s
    return ((s // 4) * 16 + m % 16) * (d // 8) + (m // 32) * 4 + s % 4, (m // 16) % 2, \
        8 * d + (s // 4) * (d // 8) + (m // 32) * 4 + s % 4


def store(code: np.ndarray, scale: np.ndarray, part: int) -> np.ndarray:
    d = code.shape[-1]
    byte, high, sbyte = places(d, part)
    out = np.zeros((*code.shape[:2], 17 * d // 2), dtype=np.uint8)
    for h in (0, 1):
        at = high == h
        out[..., byte[at]] |= code[..., at] << (4 * h)
    out[..., sbyte[:, ::GROUP]] = scale
    return out


def load(tiles: np.ndarray, d: int, part: int):
    byte, high, sbyte = places(d, part)
    return tiles[..., byte] >> (4 * high).astype(np.uint8) & 15, tiles[..., sbyte[:, ::GROUP]]


def write(code, scale, table, lengths, start, rows, index=None, max_rows=None):
    """Appends rows [rows][kv-heads][d] to token-major codes and scales in place."""
    cap = table.shape[1] * PAGE
    for b, L in enumerate(lengths):
        n = min(start[b + 1] - start[b], cap - L, 1 << 30 if max_rows is None else max_rows)
        for t in range(n):
            r = start[b] + t if index is None else index[start[b] + t]
            page = table[b, (L + t) // PAGE]
            if 0 <= r < len(rows) and 0 <= page < len(code):
                code[page, :, (L + t) % PAGE], scale[page, :, (L + t) % PAGE] = encode(rows[r])


def cached(code, scale, table_row, n):
    """The first n cached vectors [n][kv-heads][d] of one sequence, in float64."""
    ids = table_row[:-(-n // PAGE)]
    v = decode(code[ids], scale[ids])
    return v.transpose(0, 2, 1, 3).reshape(-1, *v.shape[1::2])[:n]
