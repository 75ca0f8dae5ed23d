"""Plain 64-bit numpy form of a step with drafted tokens over the 8-bit cache
(readme_rotary, readme_kv_append, readme_attention_kv_tree,
readme_verify_drafts), row by row.  Test infrastructure; shares no code with the
library.
"""
from __future__ import annotations

import math

import numpy as np

from . import kv_cache as kc


def rotary_freqs(rot, theta=10000.0, scaling="plain", factor=1.0, trained_len=0.0, low=1.0,
                 high=32.0):
    f = np.array([theta ** (-2.0 * i / rot) for i in range(rot // 2)])
    if scaling == "linear":
        f = f / factor
    elif scaling == "banded":
        n = trained_len * f / (2 * math.pi)
        g = np.clip((n - low) / (high - low), 0.0, 1.0)
        f = f * (g + (1 - g) / factor)
    return f


def rotary(x, pos, freqs, layout="half", amplitude=1.0, inverse=False):
    """x [T][H][D] float64; the angle is one rounded product, as stated."""
    y = x.copy()
    rot = 2 * len(freqs)
    for t in range(x.shape[0]):
        angle = float(pos[t]) * freqs
        c, s = amplitude * np.cos(angle), amplitude * np.sin(angle)
        if inverse:
            s = -s
        a = slice(0, rot // 2) if layout == "half" else slice(0, rot, 2)
        b = slice(rot // 2, rot) if layout == "half" else slice(1, rot, 2)
        y[t, :, a] = x[t, :, a] * c - x[t, :, b] * s
        y[t, :, b] = x[t, :, b] * c + x[t, :, a] * s
    return y


def bits(parents) -> list:
    """Python integers: row i's bits are its ancestors' and its own."""
    out = []
    for i, q in enumerate(parents):
        out.append((out[q] if q >= 0 else 0) | (1 << i))
    return out


def words(masks, n_words) -> np.ndarray:
    """Rows' bits as the call's int64 [T][words]."""
    m = (1 << 64) - 1
    return np.array([[(b >> (64 * w)) & m for w in range(n_words)] for b in masks],
                    np.uint64).reshape(len(masks), n_words).view(np.int64)


def depths(parents) -> list:
    d = []
    for q in parents:
        d.append(d[q] + 1 if q >= 0 else 0)
    return d


def attention_tree(cache, q, offsets, lens, table, masks, scale, pos=None, window=0, n_words=1,
                   fill=0.0):
    """q [T][H][D] float64, masks[t] python integers.  Returns (o, vmax, zabs) as
    kv_cache.attention."""
    codes, scales = cache["codes"], cache["scales"]
    nb, Hk, _, _, D = codes.shape
    T, H, _ = q.shape
    G = H // Hk
    o = np.full((T, H, D), fill)
    vmax, zabs = np.zeros((T, H)), np.zeros((T, H))
    for r in range(len(lens)):
        n, ln = int(offsets[r + 1] - offsets[r]), int(lens[r])
        first = ln - n
        where = [kc.block_of(table, nb, r, j) for j in range(max(ln, 0))]
        for i in range(n):
            t = int(offsets[r]) + i
            p = max(first + i if pos is None else int(pos[t]), first)
            js = []
            for j in range(max(ln, 0)):
                if where[j] < 0:
                    continue
                if j < first:
                    ok = window == 0 or j > p - window
                else:
                    ok = j - first < 64 * n_words and (masks[t] >> (j - first)) & 1
                if ok:
                    js.append(j)
            o[t] = 0.0
            if not js:
                continue
            b = np.array([where[j] for j in js])
            sl = np.array([j % kc.BLOCK for j in js])
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


def _counted(x):
    return np.where(x > 0, x, 0.0)


def verify(offsets, tokens, parent, p, q, u, distinct=False, max_rows=1024):
    """(path [T], accepted [R], token [R], margin): margin is how near, relative to
    the compared sums, any decision came to falling otherwise."""
    T, V = p.shape
    R = len(offsets) - 1
    path = np.full(T, -1, np.int64)
    accepted, token = np.zeros(R, np.int64), np.full(R, -1, np.int64)
    margin = math.inf
    for r in range(R):
        o, n = int(offsets[r]), int(offsets[r + 1] - offsets[r])
        if n == 0:
            continue
        path[o] = 0
        node, t, a, gone = 0, _counted(p[o]), 1.0, []
        i = 1
        while i < min(n, max_rows):
            if int(parent[o + i]) != node:
                i += 1
                continue
            x = int(tokens[o + i])
            if q is None:
                qq = np.zeros(V)
                if 0 <= x < V:
                    qq[x] = 1.0
            else:
                qq = _counted(q[o + node]).copy()
                if distinct:
                    qq[gone] = 0.0
            qx, tx = (qq[x], t[x]) if 0 <= x < V else (0.0, 0.0)
            left = float(u[o + i]) * a * qx
            if max(left, tx) > 0:
                margin = min(margin, abs(left - tx) / max(left, tx))
            if left < tx:
                accepted[r] += 1
                path[o + accepted[r]] = i
                node, t, a, gone = i, _counted(p[o + i]), 1.0, []
            else:
                rest = t.copy()
                if q is None:
                    if 0 <= x < V:
                        rest[x] = 0.0
                else:
                    rest = np.maximum(t - a * qq, 0.0)
                if not rest.sum() > 0:
                    break
                t = rest
                if 0 <= x < V:
                    gone.append(x)
                s = 1.0
                if distinct and q is not None:
                    qq[gone] = 0.0
                    s = qq.sum()
                a = t.sum() / s if s > 0 else 0.0
            i += 1
        run = np.cumsum(t)
        border = float(u[o]) * run[-1]
        above = np.nonzero(run > border)[0]
        if run[-1] > 0:
            token[r] = above[0]
            margin = min(margin, float(np.abs(run - border).min() / run[-1]) if border > 0 else 1.0)
    return path, accepted, token, margin
