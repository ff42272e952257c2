"""fp64 oracle of the calls around a cache that grows: rotary positions, rows written into the paged
cache and read back, attention of drafted trees.

TEST INFRASTRUCTURE ONLY (see kvprm_oracle). Caches are token-major numpy arrays of raw storage
words, [pages][kv-heads][16][head_dim]; ``store`` / ``load`` turn them into the pools' tile order
and back with the layout decoders of kvprm_oracle.
"""
from __future__ import annotations

import math

import numpy as np

from . import kvprm_oracle as ko

PAGE = 16
WORD = {"f32": np.uint32, "bf16": np.uint16, "fp8": np.uint8}


def _order(d: int, eb: int, part: int) -> np.ndarray:
    """order[i] = token-major index of a stored tile's element i."""
    dec = ko.v_tile_to_tokens if part else ko.k_tile_to_tokens
    at = dec(np.arange(PAGE * d), PAGE, d, eb).reshape(-1)  # token-major place -> stored index
    order = np.empty_like(at)
    order[at] = np.arange(PAGE * d)
    return order


def store(tok: np.ndarray, part: int) -> np.ndarray:
    p, h, _, d = tok.shape
    out = tok.reshape(p, h, -1)[:, :, _order(d, tok.itemsize, part)]
    return np.ascontiguousarray(out).reshape(tok.shape)


def load(stored: np.ndarray, part: int) -> np.ndarray:
    p, h, _, d = stored.shape
    out = np.empty((p, h, PAGE * d), dtype=stored.dtype)
    out[:, :, _order(d, stored.itemsize, part)] = stored.reshape(p, h, -1)
    return out.reshape(stored.shape)


# ------------------------------------------------------------------------------ rounding


def to_bf16(x: np.ndarray) -> np.ndarray:
    """fp32 values -> bf16 words, nearest even (NaN stays NaN)."""
    u = np.asarray(x, dtype=np.float32).view(np.uint32)
    out = ((u.astype(np.uint64) + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint16)
    return np.where(np.isnan(x), np.uint16(0x7FC0), out)


def to_e4m3(x: np.ndarray) -> np.ndarray:
    """float64 values, |x| <= 448 or not finite -> e4m3fn codes, nearest even; not finite: NaN."""
    codes = np.arange(0x7F, dtype=np.uint8)
    vals = ko.e4m3fn_to_f64(codes)
    a = np.abs(np.where(np.isfinite(x), x, 0.0))
    hi = np.minimum(np.searchsorted(vals, a), len(vals) - 1)
    lo = np.maximum(hi - 1, 0)
    up, down = vals[hi] - a, a - vals[lo]
    pick = np.where((up < down) | ((up == down) & (codes[hi] % 2 == 0)), hi, lo).astype(np.uint8)
    return np.where(np.isfinite(x), pick | np.where(np.signbit(x), 0x80, 0).astype(np.uint8), 0x7F)


def power(x: float) -> float:
    """The smallest power of two >= x (x > 0)."""
    m, e = math.frexp(x)
    return 2.0 ** (e - 1 if m == 0.5 else e)


# ------------------------------------------------------------------------------ rotary


def frequencies(n, theta, scaling="none", factor=1.0, trained=0.0, low=1.0, high=32.0):
    """Angle per position of the n / 2 pairs."""
    out = []
    for i in range(n // 2):
        f = theta ** (-2 * i / n)
        if scaling == "linear":
            f = f / factor
        if scaling == "base" and n > 2:
            f = (theta * factor ** (n / (n - 2))) ** (-2 * i / n)
        if scaling == "parts":
            turns = trained / (2 * math.pi / f)  # trained length over wavelength
            w = 0.0 if turns <= low else 1.0 if turns >= high else (turns - low) / (high - low)
            f = (1 - w) * f / factor + w * f
        if scaling == "ramp":
            def at(t):
                return n * math.log(trained / (t * 2 * math.pi)) / (2 * math.log(theta))
            a, b = max(math.floor(at(high)), 0), min(math.ceil(at(low)), n - 1)
            w = 1 - min(max((i - a) / max(b - a, 0.001), 0), 1)
            f = (1 - w) * f / factor + w * f
        out.append(f)
    return np.array(out)


def rotary(x, pos, freq, layout="half", magnitude=1.0, transpose=False):
    """x [rows][heads][d]; the first 2 len(freq) dims of each head are rotated."""
    n = 2 * len(freq)
    phi = np.asarray(pos, dtype=np.float64)[:, None] * freq
    turn = magnitude * np.exp((-1j if transpose else 1j) * phi)[:, None]
    lo, hi = (slice(0, n // 2), slice(n // 2, n)) if layout == "half" else (slice(0, n, 2), slice(1, n, 2))
    y = np.array(x, dtype=np.float64)
    z = (y[..., lo] + 1j * y[..., hi]) * turn
    y[..., lo], y[..., hi] = z.real, z.imag
    return y


# ------------------------------------------------------------------------------ cache rows


def write(tok, scale, dtype, table, lengths, start, rows, index=None, max_rows=None):
    """Appends rows [rows][kv-heads][d] (fp32 or bf16 values as float32) to token-major raw tiles
    `tok` and, for fp8, their scales [pages][kv-heads], in place."""
    pages, nkv = tok.shape[:2]
    cap = table.shape[1] * PAGE
    for b, L in enumerate(lengths):
        n = start[b + 1] - start[b]
        n = min(n, cap - L, n if max_rows is None else max_rows)
        for p in range(L // PAGE, -(-(L + n) // PAGE) if n > 0 else 0):
            page = table[b, p]
            if page < 0 or page >= pages:
                continue
            new = {}
            for s in range(PAGE):
                t = p * PAGE + s - L
                if 0 <= t < n:
                    r = start[b] + t if index is None else index[start[b] + t]
                    if 0 <= r < len(rows):
                        new[s] = rows[r]
            if not new:
                continue
            old = range(max(0, min(PAGE, L - p * PAGE)))
            for j in range(nkv):
                if dtype != "fp8":
                    for s, v in new.items():
                        v = v[j].astype(np.float32)
                        tok[page, j, s] = to_bf16(v) if dtype == "bf16" else v.view(np.uint32)
                    continue
                a = np.abs(np.stack([v[j] for v in new.values()]).astype(np.float64))
                a = np.max(np.where(np.isfinite(a), a, 0))
                unit = max(power(a / 448) if a > 0 else 0.0, 2.0 ** -100)
                if len(old):
                    unit = max(unit, power(float(scale[page, j])))
                    if unit != scale[page, j]:
                        was = ko.e4m3fn_to_f64(tok[page, j, :len(old)]) * np.float64(scale[page, j])
                        tok[page, j, :len(old)] = to_e4m3(was / unit)
                for s, v in new.items():
                    tok[page, j, s] = to_e4m3(v[j].astype(np.float64) / unit)
                scale[page, j] = unit


def cached(tok, scale, dtype, table_row, n):
    """The first n cached vectors [n][kv-heads][d] of one sequence, in float64."""
    ids = table_row[:-(-n // PAGE)]
    v = tok[ids].view(np.float32).astype(np.float64) if dtype == "f32" else ko.decode_storage(tok[ids], dtype)
    if dtype == "fp8":
        v = v * scale[ids].astype(np.float64)[..., None, None]
    return v.transpose(0, 2, 1, 3).reshape(-1, *v.shape[1::2])[:n]


# ------------------------------------------------------------------------------ drafted trees


def tree_attention(q, k, v, ck, cv, sees):
    """One sequence: q [T][n_q][d], drafted k, v [T][n_kv][d], cached ck, cv [L][n_kv][d], sees [T][T]
    (drafted token i attends to drafted token j). A token that attends to nothing gets zeros."""
    T, nq, d = q.shape
    g = nq // k.shape[1]
    o = np.zeros((T, nq, d))
    for i in range(T):
        js = np.flatnonzero(sees[i])
        for h in range(nq):
            K = np.concatenate([ck[:, h // g], k[js, h // g]])
            V = np.concatenate([cv[:, h // g], v[js, h // g]])
            if len(K):
                with np.errstate(invalid="ignore"):
                    s = K @ q[i, h] / math.sqrt(d)
                    p = np.exp(s - np.max(s))
                    o[i, h] = p @ V / p.sum()
    return o
