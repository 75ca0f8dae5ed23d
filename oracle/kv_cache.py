"""Plain 64-bit numpy form of the 8-bit key/value cache (readme_kv_write,
readme_kv_read, readme_attention_kv): token by token and row by row, on arrays
of code values.  Test infrastructure; shares no code with the library.

A cache is a dict: `codes` float64 [n_blocks][Hk][2][64][D] (code values),
`scales` float32 [n_blocks][Hk][2].
"""
from __future__ import annotations

import math

import numpy as np

BLOCK = 64
FLOOR = 2.0 ** -100
QMAX = {"i8": 127.0, "e4m3": 448.0}


def e4m3_values() -> np.ndarray:
    """Value of every e4m3 byte: sign, 4 exponent bits (bias 7), 3 mantissa
    bits; 0x7f and 0xff are NaN."""
    out = np.empty(256)
    for b in range(256):
        e, m = (b >> 3) & 15, b & 7
        v = m * 2.0 ** -9 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        out[b] = math.nan if (b & 127) == 127 else (-v if b & 128 else v)
    return out


def nearest(kt: str, q: np.ndarray) -> np.ndarray:
    """The code nearest to each q, ties to the even one, largest magnitude
    QMAX."""
    if kt == "i8":
        return np.clip(np.rint(q), -127.0, 127.0)
    grid = np.sort(e4m3_values()[:127])               # 0 .. 448, index = byte
    a = np.minimum(np.abs(q), 448.0)
    hi = np.clip(np.searchsorted(grid, a), 1, 126)
    lo = hi - 1
    up, down = grid[hi] - a, a - grid[lo]
    pick = np.where(up < down, hi, np.where(up > down, lo, np.where(hi % 2 == 0, hi, lo)))
    return np.copysign(grid[pick], q)


def new_cache(n_blocks: int, Hk: int, D: int) -> dict:
    return {"codes": np.zeros((n_blocks, Hk, 2, BLOCK, D)),
            "scales": np.zeros((n_blocks, Hk, 2), np.float32)}


def to_bytes(kt: str, codes: np.ndarray) -> np.ndarray:
    """Code values to the library's bytes [n_blocks][Hk][2][64 D]."""
    n, Hk, _, _, D = codes.shape
    if kt == "i8":
        b = (codes + 128).astype(np.uint8)
    else:
        vals = e4m3_values()
        order = np.argsort(np.abs(vals[:127]))
        mag = order[np.searchsorted(np.abs(vals[:127])[order], np.abs(codes))]
        b = (mag + 128 * np.signbit(codes)).astype(np.uint8)
    k = b[:, :, 0].reshape(n, Hk, 2, 32, D // 16, 16).transpose(0, 1, 2, 4, 3, 5)
    v = b[:, :, 1].reshape(n, Hk, 2, 32, D).transpose(0, 1, 2, 4, 3)
    return np.stack([k.reshape(n, Hk, BLOCK * D), v.reshape(n, Hk, BLOCK * D)], 2)


def from_bytes(kt: str, raw: np.ndarray, D: int) -> np.ndarray:
    n, Hk = raw.shape[:2]
    x = raw.astype(np.float64) - 128 if kt == "i8" else e4m3_values()[raw]
    k = x[:, :, 0].reshape(n, Hk, 2, D // 16, 32, 16).transpose(0, 1, 2, 4, 3, 5)
    v = x[:, :, 1].reshape(n, Hk, 2, D, 32).transpose(0, 1, 2, 4, 3)
    return np.stack([k.reshape(n, Hk, BLOCK, D), v.reshape(n, Hk, BLOCK, D)], 2)


def block_of(table: np.ndarray, n_blocks: int, r: int, p: int) -> int:
    if p < 0 or p // BLOCK >= table.shape[1]:
        return -1
    b = int(table[r, p // BLOCK])
    return b if 0 <= b < n_blocks else -1


def write(kt, cache, k, v, offsets, lens, table) -> None:
    """k, v [T][Hk][D] float64."""
    codes, scales = cache["codes"], cache["scales"]
    nb, Hk = codes.shape[:2]
    for r in range(len(lens)):
        n = int(offsets[r + 1] - offsets[r])
        first = int(lens[r]) - n
        groups = {}
        for i in range(n):
            p = first + i
            b = block_of(table, nb, r, p)
            if b >= 0:
                groups.setdefault((p // BLOCK, b), []).append((p % BLOCK, int(offsets[r]) + i))
        for (_, b), rows in groups.items():
            start = rows[0][0]
            for half, src in ((0, k), (1, v)):
                for h in range(Hk):
                    x = np.stack([src[t, h] for _, t in rows])
                    old = float(scales[b, h, half])
                    finite = np.isfinite(x).all()
                    if not finite or (start > 0 and not (old > 0 and math.isfinite(old))):
                        scales[b, h, half] = np.nan
                        for slot, _ in rows:
                            codes[b, h, half, slot] = 0.0
                        continue
                    need = float(np.float32(np.abs(x).max() / QMAX[kt]))
                    if start == 0:
                        s = max(need, FLOOR)
                    else:
                        s = old
                        while s < need:
                            s *= 2.0
                        codes[b, h, half, :start] = nearest(kt, codes[b, h, half, :start] * (old / s))
                    scales[b, h, half] = s
                    for (slot, _), row in zip(rows, x):
                        codes[b, h, half, slot] = nearest(kt, row / s)


def read(cache, T, offsets, lens, table, fill=0.0):
    """(k, v) [T][Hk][D] float64; rows of no request hold `fill`."""
    codes, scales = cache["codes"], cache["scales"]
    nb, Hk, _, _, D = codes.shape
    out = np.full((2, T, Hk, D), fill)
    for r in range(len(lens)):
        n = int(offsets[r + 1] - offsets[r])
        for i in range(n):
            p = int(lens[r]) - n + i
            b = block_of(table, nb, r, p)
            t = int(offsets[r]) + i
            out[:, t] = 0.0
            if b >= 0:
                x = codes[b, :, :, p % BLOCK] * scales[b].astype(np.float64)[..., None]
                out[:, t] = x.transpose(1, 0, 2)
    return out[0], out[1]


def attention(cache, q, offsets, lens, table, scale, causal=True, window=0, fill=0.0):
    """q [T][H][D] float64.  Returns (o [T][H][D], bound pieces): per row and
    head the largest |v| it sees and the largest sum of |q||k| * scale."""
    codes, scales = cache["codes"], cache["scales"]
    nb, Hk, _, _, D = codes.shape
    T, H, _ = q.shape
    G = H // Hk
    o = np.full((T, H, D), fill)
    vmax, zabs = np.zeros((T, H)), np.zeros((T, H))
    for r in range(len(lens)):
        n, ln = int(offsets[r + 1] - offsets[r]), int(lens[r])
        where = [block_of(table, nb, r, j) for j in range(max(ln, 0))]
        for i in range(n):
            t, p = int(offsets[r]) + i, ln - n + i
            js = [j for j in range(max(ln, 0)) if where[j] >= 0 and (not causal or j <= p) and
                  (window == 0 or j > p - window)]
            o[t] = 0.0
            if not js:
                continue
            b = np.array([where[j] for j in js])
            sl = np.array([j % BLOCK for j in js])
            for h in range(Hk):
                kk = codes[b, h, 0, sl] * scales[b, h, 0].astype(np.float64)[:, None]
                vv = codes[b, h, 1, sl] * scales[b, h, 1].astype(np.float64)[:, None]
                for g in range(h * G, (h + 1) * G):
                    z = kk @ q[t, g] * scale
                    w = np.exp(z - z.max())
                    o[t, g] = w @ vv / w.sum()
                    vmax[t, g] = np.abs(vv).max()
                    zabs[t, g] = (np.abs(kk) @ np.abs(q[t, g])).max() * scale
    return o, vmax, zabs
