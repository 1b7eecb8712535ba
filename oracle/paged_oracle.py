"""Rotary positions, the paged 4-bit cache and attention over it, in numpy.

Definitions only (test infrastructure; imports nothing from the library).  What
the library computes in fp32 with fixed roundings (a key's rotation before it is
held, a group's scale, minimum and codes) is restated with the same roundings,
so that held bytes compare bit for bit; everything else is fp64.
"""
from __future__ import annotations

import math

import numpy as np

F32 = np.float32


# --- rotary positions --------------------------------------------------------

def frequencies(rot_dim: int, base: float = 500000.0, scaling: str = "none", factor: float = 1.0,
                original: float = 8192.0, low: float = 1.0, high: float = 4.0, beta_fast: float = 32.0,
                beta_slow: float = 1.0) -> np.ndarray:
    """Radians per position of every pair, for the scalings of reskv_rope_config."""
    i = np.arange(rot_dim // 2, dtype=np.float64)
    if scaling == "base":
        base = base * factor ** (rot_dim / (rot_dim - 2))
    f = base ** (-2.0 * i / rot_dim)
    if scaling in ("none", "base"):
        return f
    if scaling == "linear":
        return f / factor
    if scaling == "wavelength":
        turns = original * f / (2 * math.pi)
        keep = np.clip((turns - low) / (high - low), 0, 1)
    else:
        pair = lambda b: rot_dim * math.log(original / (b * 2 * math.pi)) / (2 * math.log(base))  # noqa: E731
        first = max(0, math.floor(pair(beta_fast)))
        last = max(first + 1e-3, min(rot_dim - 1, math.ceil(pair(beta_slow))))
        keep = 1 - np.clip((i - first) / (last - first), 0, 1)
    return f * keep + f / factor * (1 - keep)


def table(n: int, f: np.ndarray, magnitude: float = 1.0) -> np.ndarray:
    a = np.arange(n, dtype=np.float64)[:, None] * f
    return magnitude * np.stack([np.cos(a), np.sin(a)], -1)


def rotate(x: np.ndarray, cs: np.ndarray, interleaved: bool, backward: bool = False) -> np.ndarray:
    """Rows x [T, H, d] turned by cs [T, R / 2, 2] in x's and cs's type (each operation rounded)."""
    R = 2 * cs.shape[1]
    c, s = cs[:, None, :, 0], cs[:, None, :, 1]
    if backward:
        s = -s
    y = x.copy()
    ia = slice(0, R, 2) if interleaved else slice(0, R // 2)
    ib = slice(1, R, 2) if interleaved else slice(R // 2, R)
    a, b = x[..., ia], x[..., ib]
    y[..., ia] = a * c - b * s
    y[..., ib] = b * c + a * s
    return y


# --- held rows ---------------------------------------------------------------

def bf16_bits(x: np.ndarray) -> np.ndarray:
    """fp32 -> bf16 bit patterns, round to nearest even (uint32)."""
    u = np.ascontiguousarray(x, F32).view(np.uint32)
    r = ((u + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint32)
    return np.where(np.isnan(x), np.uint32(0x7FC0), r)


def bf16_value(bits: np.ndarray) -> np.ndarray:
    return (np.asarray(bits, np.uint32) << 16).view(F32)


def hold(x: np.ndarray, group: int):
    """fp32 rows [.., d] -> codes [.., d], bf16 bits of scales and minima [.., d / group]."""
    y = np.asarray(x, F32).reshape(*x.shape[:-1], x.shape[-1] // group, group)
    with np.errstate(all="ignore"):
        lo, hi = y.min(-1), y.max(-1)
        s16, m16 = bf16_bits((hi - lo) / F32(15)), bf16_bits(lo)
        s, m = bf16_value(s16), bf16_value(m16)
        bad = ~(np.isfinite(s) & np.isfinite(m))
        flat = ~bad & (s < F32(2.0 ** -126))
        n = np.clip(np.rint((y - m[..., None]) / s[..., None]), 0, 15)
    n[bad | flat] = 0
    s16, m16 = np.where(bad, 0x7FC0, np.where(flat, 0, s16)), np.where(bad, 0x7FC0, m16)
    return n.reshape(x.shape).astype(np.uint8), s16.astype(np.uint16), m16.astype(np.uint16)


def held_value(n: np.ndarray, s16: np.ndarray, m16: np.ndarray) -> np.ndarray:
    """What codes stand for, fp64."""
    group = n.shape[-1] // s16.shape[-1]
    s, m = (np.repeat(bf16_value(b).astype(np.float64), group, -1) for b in (s16, m16))
    return n * s + m


def tile_bytes(d: int, group: int) -> int:
    return 2 * (8 * d + 64 * (d // group))


def put_row(page: np.ndarray, head: int, slot: int, d: int, group: int, which: int, n, s16, m16):
    """Write one row into page [heads, bytes] (uint8): which 0 = K, 1 = V."""
    ng, row, tile = d // group, slot % 16, slot // 16
    t = page[head, tile * tile_bytes(d, group):(tile + 1) * tile_bytes(d, group)]
    if which == 0:
        for x in range(d):
            w = x // 8
            byte = row * (d // 2) + 4 * ((w % 4) * (d // 32) + w // 4) + (x % 8) // 2
            t[byte] = (t[byte] & (0xF0 if x % 2 == 0 else 0x0F)) | (int(n[x]) << (4 * (x % 2)))
        at = 8 * d
    else:
        r = row // 2
        z = 2 * (r % 4) if d == 128 else 4 * (r // 2 % 2)
        for x in range(d):
            c, g, i = x // 32, x % 32 // 4, x % 4
            byte = 8 * d + 64 * ng + r * d + (g ^ z) * (d // 8) + 4 * c + 2 * (row % 2) + i // 2
            t[byte] = (t[byte] & (0xF0 if i % 2 == 0 else 0x0F)) | (int(n[x]) << (4 * (i % 2)))
        at = 16 * d + 64 * ng
    meta = t[at + row * 4 * ng:at + (row + 1) * 4 * ng]
    meta[:] = np.concatenate([s16, m16]).astype("<u2").view(np.uint8)


# --- attention ---------------------------------------------------------------

def attend(q: np.ndarray, k: np.ndarray, v: np.ndarray, per: int, scale: float, window: int = 0):
    """q [n, Hq, d] the newest of the len tokens of k, v [Hkv, len, d]: o [n, Hq, d], lse [n, Hq], and for a
    tolerance the largest scale * sum |q k| and |v| any query sees."""
    n, Hq, d = q.shape
    length = k.shape[1]
    o, lse = np.zeros((n, Hq, d)), np.full((n, Hq), -np.inf)
    xmax, vmax = np.zeros((n, Hq)), np.zeros((n, Hq))
    for i in range(n):
        p = length - n + i
        t0 = max(0, p - window + 1) if window else 0
        if p < 0:
            continue
        for h in range(Hq):
            kk, vv = k[h // per, t0:p + 1], v[h // per, t0:p + 1]
            x = scale * (kk @ q[i, h])
            top = x.max()
            w = np.exp(x - top)
            o[i, h] = (w @ vv) / w.sum()
            lse[i, h] = top + math.log(w.sum())
            xmax[i, h] = scale * (np.abs(kk) @ np.abs(q[i, h])).max()
            vmax[i, h] = np.abs(vv).max()
    return o, lse, xmax, vmax
