"""The attention operators' definitions in numpy: rotary positions, the 4-bit form of keys and values and its pages, attention.

Test infrastructure only; written from the formulas in include/liquidgemm.h, element by element where that is affordable.
"""
from __future__ import annotations

import math

import numpy as np

F16, BF16 = "float16", "bfloat16"
UNIT = {F16: 2.0 ** -11, BF16: 2.0 ** -8}  # largest relative error of rounding to the type


def round_to(x, dtype):
    """float32 / float64 -> the type's values (ties to even), as float32.  (BF16 by integer arithmetic on FP32.)"""
    x = np.asarray(x, dtype=np.float32)
    if dtype == F16:
        with np.errstate(over="ignore"):
            return x.astype(np.float16).astype(np.float32)
    bits = x.view(np.uint32).astype(np.uint64)
    up = (bits + 0x7FFF + ((bits >> 16) & 1)) & 0xFFFF0000
    return np.where(np.isfinite(x), up.astype(np.uint32).view(np.float32), x)


# ------------------------------------------------------------------------------ rotary positions
def rope_table(positions, rot, base=10000.0, scaling=None, factor=1.0, original=0):
    half = rot // 2
    if scaling == "ntk":
        base = base * factor ** (rot / (rot - 2))
    freq = np.array([base ** (-2 * i / rot) for i in range(half)])
    magnitude = 1.0
    if scaling == "linear":
        freq = freq / factor
    if scaling == "yarn":
        turns_at = lambda turns: rot * math.log(original / (2 * math.pi * turns)) / (2 * math.log(base))
        low, high = max(math.floor(turns_at(32)), 0), min(math.ceil(turns_at(1)), rot - 1)
        if high <= low:
            high = low + 0.001
        mix = np.clip((np.arange(half) - low) / (high - low), 0, 1)
        freq = freq * (1 - mix) + freq / factor * mix
        magnitude = 0.1 * math.log(factor) + 1
    angle = np.arange(positions)[:, None] * freq
    return np.concatenate((np.cos(angle), np.sin(angle)), 1) * magnitude


def rope(x, positions, table, interleaved=False, weight=None, eps=1e-6, dtype=np.float32):
    """x [T, H, D], unrounded result in `dtype` arithmetic (every operation rounded to it)."""
    y = x.astype(dtype)
    if weight is not None:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + dtype(eps)) * weight.astype(dtype)
    rot = table.shape[1]
    half = rot // 2
    row = table[positions].astype(dtype)[:, None]
    c, s = row[..., :half], row[..., half:]
    i = np.arange(half)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    out = y.copy()
    out[..., a] = y[..., a] * c - y[..., b] * s
    out[..., b] = y[..., b] * c + y[..., a] * s
    return out


# ------------------------------------------------------------------------------- the 4-bit form
def quantise(x):
    """x [..., D] of FP16 or BF16 values -> codes uint8 [..., D], scale float32 [...], zero point uint8 [...]; exact arithmetic."""
    x = np.asarray(x, dtype=np.float64)
    lo, hi = np.minimum(x.min(-1), 0), np.maximum(x.max(-1), 0)
    r = (hi - lo).astype(np.float32) / np.float32(15)
    m, e = np.frexp(r.astype(np.float64))
    s = np.maximum(np.ldexp(np.rint(np.ldexp(m, 12)), e - 12), 2.0 ** -100)
    z = np.rint(-lo / s)
    codes = np.clip(np.rint(x / s[..., None]) + z[..., None], 0, 15)
    return codes.astype(np.uint8), s.astype(np.float32), z.astype(np.uint8)


def dequantise(codes, s, z):
    return (codes.astype(np.float64) - z.astype(np.float64)[..., None]) * s.astype(np.float64)[..., None]


def store(cache, page_size, slot, head, codes, s, z, value):
    """One vector into its page: cache uint8 [pages, kv_heads, page_size * (D + 8)]."""
    D = len(codes)
    at = cache[slot // page_size, head]
    j = slot % page_size
    for d in range(D):
        if value:
            width = D // 16
            group, inside = divmod(d, width)
            byte = page_size * D // 2 + (j // 4) * 2 * D + group * (D // 8) + (j % 4 // 2) * (D // 16) + inside // 4 * 4 + j % 2 * 2 + inside % 4 // 2
        else:
            byte = j * D // 2 + d // 2
        keep = 0xF0 if d % 2 == 0 else 0x0F
        at[byte] = (at[byte] & keep) | (codes[d] << (4 * (d % 2)))
    word = np.uint32(np.float32(s).view(np.uint32)) | np.uint32(z)
    first = page_size * D + (4 * page_size if value else 0) + 4 * j
    at[first:first + 4] = np.array([word], dtype="<u4").view(np.uint8)


def write(cache, page_size, slots, k, v):
    for x, value in ((k, False), (v, True)):
        codes, s, z = quantise(x)
        for t, slot in enumerate(slots):
            if 0 <= slot < cache.shape[0] * page_size:
                for h in range(x.shape[1]):
                    store(cache, page_size, int(slot), h, codes[t, h], s[t, h], z[t, h], value)


# ------------------------------------------------------------------------------------ attention
def attention(q, k, v, scale, limits):
    """q [n, Hq, D], k, v [len, Hkv, D], limits [n]: keys that each query sees.  Returns the result and sum_j p_j |v_j| (what the
    weights' rounding errors multiply), FP64."""
    n, Hq, D = q.shape
    group = Hq // k.shape[1]
    out, spread = np.zeros((2, n, Hq, D))
    q, k, v = (np.asarray(x, dtype=np.float64) for x in (q, k, v))
    for h in range(Hq):
        scores = q[:, h] @ k[:, h // group].T * scale
        for i in range(n):
            seen = int(min(max(limits[i], 0), len(k)))
            if seen:
                x = scores[i, :seen]
                p = np.exp(x - x.max())
                p /= p.sum()
                out[i, h] = p @ v[:seen, h // group]
                spread[i, h] = p @ np.abs(v[:seen, h // group])
    return out, spread
