"""The attention layers' serving operators in fp64 -- TEST INFRASTRUCTURE ONLY (the parity oracle of
``gdn_qk_norm_rope``, ``gdn_kv_append`` and ``gdn_attention_paged``; only tests/ use it).

Written from the definitions, token by token where positions and pages come in: nothing is shared with the HIP path.

    norm      y = x w / sqrt(mean(x^2) + eps)
    rotation  (y_a, y_b) -> (y_a cos t - y_b sin t, y_b cos t + y_a sin t),  t = position * inv_freq[i]
    cache     position p of sequence s: page table[s, p // page], slot p % page, of [n_pages, H_kv, page, d]
    e4m3      one scale per (page, head), the smallest power of two s >= 2^-100 with |x| <= 448 s
"""
from __future__ import annotations

import numpy as np


def norm(x, w, eps):
    """x [..., d] over its last axis (w None: x itself)."""
    x = np.asarray(x, dtype=np.float64)
    return x if w is None else x * np.asarray(w, dtype=np.float64) / np.sqrt((x * x).mean(-1, keepdims=True) + eps)


def rotate(x, pos, inv_freq, interleaved=False):
    """x [T, heads, d] at positions pos [T]; inv_freq [r / 2]: the first r channels rotate."""
    y = np.array(x, dtype=np.float64)
    if inv_freq is None:
        return y
    f = np.asarray(inv_freq, dtype=np.float64)
    for i in range(len(f)):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + len(f))
        t = (np.asarray(pos, dtype=np.float64) * f[i])[:, None]
        u, v = np.array(x[..., a], dtype=np.float64), np.array(x[..., b], dtype=np.float64)
        y[..., a], y[..., b] = u * np.cos(t) - v * np.sin(t), v * np.cos(t) + u * np.sin(t)
    return y


def spans(B, T, cu=None):
    """(first row, rows) of every sequence's new tokens; offsets clamped into a nondecreasing partition of [0, T]."""
    if cu is None:
        return [(b * T, T) for b in range(B)]
    out, at = [], 0
    for c in list(cu)[1:]:
        end = min(max(int(c), at), T)
        out.append((at, end - at))
        at = end
    return out


def e4m3(y):
    """Nearest e4m3 value, ties to the even one (values up to 448); NaN stays."""
    y = np.asarray(y, dtype=np.float64)
    with np.errstate(divide="ignore", invalid="ignore"):
        step = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(y), 2.0 ** -6))) - 3)
    return np.where(np.isfinite(y), np.round(y / step) * step, y)


def power_scale(amax):
    s = 2.0 ** -100
    while amax > 448 * s:
        s *= 2
    return s


def append(cache, scale, table, lens, rows, cu, B, T, page):
    """Rows [B T, H_kv, d] (normed and rotated, or values) into cache [n_pages, H_kv, page, d] (values that the
    codes stand for over the scale; updated in place) and scale [n_pages, H_kv] (None: not scaled, not rounded)."""
    n_pages, max_pages = cache.shape[0], np.shape(table)[1]
    for s, (row, n) in enumerate(spans(B, T, cu)):
        groups = {}
        for i in range(n):
            p = int(lens[s]) - n + i
            if 0 <= p < max_pages * page and 0 <= table[s][p // page] < n_pages:
                groups.setdefault(p // page, []).append((p % page, row + i))
        for b, slots in groups.items():
            at = int(table[s][b])
            for h in range(cache.shape[1]):
                x = np.array([rows[r, h] for _, r in slots])
                if scale is not None:
                    x = np.where(np.isfinite(x), x, np.nan)
                    new, held = power_scale(np.nanmax(np.abs(np.append(x, 0.0)))), slots[0][0]
                    if held and scale[at, h] >= new:
                        new = scale[at, h]
                    elif held:
                        cache[at, h, :held] = e4m3(cache[at, h, :held] * scale[at, h] / new)
                    scale[at, h] = new
                    x = e4m3(x / new)
                for (slot, _), y in zip(slots, x):
                    cache[at, h, slot] = y


def attention(q, k_cache, v_cache, table, lens, cu, B, T, sc):
    """q [B T, H, d]; caches [n_pages, H_kv, page, d] as the values they stand for.  Returns (o, a), a the same sums
    with |v| in the place of v (what a relative error of the weights acts on); rows of no sequence are NaN."""
    q = np.asarray(q, dtype=np.float64)
    n_pages, Hkv, page, d = k_cache.shape
    H, max_pages = q.shape[1], np.shape(table)[1]
    o, a = np.full(q.shape, np.nan), np.full(q.shape, np.nan)
    for s, (row, n) in enumerate(spans(B, T, cu)):
        have = [p for p in range(min(max(int(lens[s]), 0), max_pages * page)) if 0 <= table[s][p // page] < n_pages]
        pages, slots = np.array([table[s][p // page] for p in have], dtype=int), np.array([p % page for p in have], dtype=int)
        k, v = k_cache[pages, :, slots].astype(np.float64), v_cache[pages, :, slots].astype(np.float64)
        for i in range(n):
            m = int(np.searchsorted(np.array(have), int(lens[s]) - n + i, side="right")) if have else 0
            for h in range(H):
                if m == 0:
                    o[row + i, h] = a[row + i, h] = 0.0
                    continue
                z = sc * (k[:m, h // (H // Hkv)] @ q[row + i, h])
                w = np.exp(z - z.max())
                w /= w.sum()
                o[row + i, h] = w @ v[:m, h // (H // Hkv)]
                a[row + i, h] = w @ np.abs(v[:m, h // (H // Hkv)])
    return o, a
