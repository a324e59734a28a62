"""The packed cache in 64 bits, plainly: stored values, bounds, block selection and
attention, from their definitions (numpy; imports nothing from the package)."""
import math

import numpy as np

VALUES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
SCALES = np.array([c * 2.0 ** -17 if c < 8 else (8 + c % 8) * 2.0 ** (c // 8 - 18)
                   for c in range(0xE3)])  # up to 10240
BLOCK = 64


def nearest(x, grid):
    """Index of the nearest grid value, ties to the even index; above the grid, the last."""
    x = np.asarray(x, np.float64)
    hi = np.clip(np.searchsorted(grid, x), 1, len(grid) - 1)
    lo = hi - 1
    up, down = grid[hi] - x, x - grid[lo]
    return np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)


def stored(x):
    """Values of rows [..., dh] as the cache holds them."""
    x = np.asarray(x, np.float64)
    bad = ~np.isfinite(x).all(-1, keepdims=True)
    g = np.where(bad, 0.0, x).reshape(*x.shape[:-1], x.shape[-1] // 16, 16)
    s = SCALES[nearest(np.abs(g).max(-1, keepdims=True) / 6, SCALES)]
    y = np.where(s > 0, np.abs(g) / np.where(s > 0, s, 1.0), 0.0)
    v = (VALUES[nearest(y, VALUES)] * s * np.sign(g)).reshape(x.shape)
    return np.where(bad, np.nan, v)


def unit(a):
    """The smallest power of two u >= 2^-100 with a <= 127 u."""
    t = -100
    while a > 127 * 2.0 ** t:
        t += 1
    return 2.0 ** t


def bounds(k):
    """hi, lo [G, blocks, dh] and unit [G, blocks] of stored keys [n, G, dh]."""
    n, G, dh = k.shape
    nb = -(-n // BLOCK)
    hi, lo, u = np.zeros((G, nb, dh)), np.zeros((G, nb, dh)), np.zeros((G, nb))
    for g in range(G):
        for b in range(nb):
            rows = k[b * BLOCK:(b + 1) * BLOCK, g]
            rows = rows[np.isfinite(rows).all(1)]
            if len(rows) == 0:
                rows = np.zeros((1, dh))
            u[g, b] = unit(np.abs(rows).max())
            hi[g, b], lo[g, b] = np.ceil(rows.max(0) / u[g, b]), np.floor(rows.min(0) / u[g, b])
    return hi, lo, u


def select(q, pos, k, count):
    """Blocks [R, G, count] for q [R, H, dh] at positions pos over stored keys k [n, G, dh]."""
    R, H, dh = q.shape
    G = k.shape[1]
    hi, lo, u = bounds(k)
    out = np.full((R, G, count), -1, np.int64)
    for r in range(R):
        if pos[r] < 0:
            continue
        own = pos[r] // BLOCK
        for g in range(G):
            x = q[r, g * (H // G):(g + 1) * (H // G)].astype(np.float32)
            up, down = np.zeros(dh, np.float32), np.zeros(dh, np.float32)
            for h in x:  # in order, in 32 bits: part of the definition
                up, down = up + np.maximum(h, 0), down + np.minimum(h, 0)
            a = max(up.max(), -down.min())
            if np.isfinite(a):
                t = unit(float(a))
                P, N = np.rint(up.astype(np.float64) / t), np.rint(down.astype(np.float64) / t)
            else:
                P = N = np.zeros(dh)
            score = u[g] * (hi[g] @ P + lo[g] @ N)
            best = sorted(range(own), key=lambda b: (-score[b], b))[:count - 1]
            took = sorted(best + [own])
            out[r, g, :len(took)] = took
    return out


def attention(q, pos, k, v, blocks=None):
    """out [R, H, dh] and the rounding scales of a test: the largest |v| that a head's row
    sees and the largest sum |q k| / sqrt(dh) [R, H]."""
    R, H, dh = q.shape
    n, G = k.shape[:2]
    out, vmax, smax = np.zeros((R, H, dh)), np.zeros((R, H)), np.zeros((R, H))
    for r in range(R):
        for g in range(G):
            if blocks is None:
                js = np.arange(max(0, pos[r] + 1))
            else:
                js = np.concatenate([np.arange(b * BLOCK, min((b + 1) * BLOCK, pos[r] + 1))
                                     for b in blocks[r, g] if 0 <= b <= pos[r] // BLOCK]
                                    + [np.zeros(0, int)]).astype(int)
            if len(js) == 0:
                continue
            K, V = k[js, g], v[js, g]
            for h in range(g * (H // G), (g + 1) * (H // G)):
                x = K @ q[r, h] / math.sqrt(dh)
                if np.isnan(x).any() or np.isnan(V).any():
                    out[r, h] = np.nan
                    continue
                w = np.exp(x - x.max())
                out[r, h] = w @ V / w.sum()
                vmax[r, h] = np.abs(V).max()
                smax[r, h] = (np.abs(K) @ np.abs(q[r, h])).max() / math.sqrt(dh)
    return out, vmax, smax
