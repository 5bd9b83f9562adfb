"""Inputs and bounds shared by the tests of the paged cache's entry points."""
import numpy as np
import torch

import paper_2607_14568_amd as gdn
from oracle import paged

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}   # half a step, relative
f64 = lambda t: t.detach().cpu().double().numpy()   # noqa: E731


def normal(seed, *shape, dtype=torch.bfloat16):
    return torch.from_numpy(np.random.default_rng(seed).standard_normal(shape)).to(dtype)


def freqs(rot):
    return torch.from_numpy(10000.0 ** (-np.arange(0, rot, 2) / rot)) if rot else None


def turned(x, w, eps, pos, f, near):
    """fp64 rows of x [B,T,heads,d] as [B T, heads, d], and what a row's fp32 steps may be off by, relative to its largest
    normed value: a sum of d squares over 8 + log2(lanes) additions, a root, a quotient and two products (2^-20); an angle
    of up to half a turn rounded to fp32 (2^-24 of 2 pi / 2, under 2^-22), a few units of cos and sin (2^-22) and two
    products and a sum, each on two values: under 2^-18."""
    y = paged.norm(f64(x).reshape(-1, *x.shape[2:]), None if w is None else f64(w), eps)
    ref = paged.rotate(y, pos, None if f is None else f64(f), near)
    return ref, 2.0 ** -18 * np.abs(y).max(-1, keepdims=True)


def pages_for(lens, page, seed, extra=3, width=1):
    """A table [n, max_pages] of distinct pages in random order, -1 behind a sequence's last, and the number of pages."""
    need = [-(-max(x, 0) // page) for x in lens]
    n_pages = sum(need) + extra
    order = np.random.default_rng(seed).permutation(n_pages)
    table = np.full((len(lens), max(need) + width), -1, dtype=np.int32)
    at = 0
    for s, c in enumerate(need):
        table[s, :c] = order[at:at + c]
        at += c
    return table, n_pages


def make_cache(n_pages, Hkv, page, d, cache, seed):
    """(k, v, ks, vs) on the CPU, in the cache's type; an 8-bit cache's sizes differ by page and head."""
    out = []
    for i in range(2):
        g = np.random.default_rng(seed + i)
        x = g.standard_normal((n_pages, Hkv, page, d))
        if cache == "bf16":
            out += [torch.from_numpy(x).bfloat16(), None]
        else:
            s = 2.0 ** g.integers(-8, -4, (n_pages, Hkv))
            out += [torch.from_numpy(np.clip(x * 64, -448, 448)).to(torch.float8_e4m3fn), torch.from_numpy(s).float()]
    return out[0], out[2], out[1], out[3]


def values(cache, scale):
    """fp64 values that a cache's codes stand for."""
    return f64(cache.float()) * (1 if scale is None else f64(scale)[..., None, None])


def cuda(*ts):
    return [None if t is None else t.cuda() for t in ts]


def attend(q, cache, table, lens, cu=None, scale=None, o=None, workspace=None):
    k, v, ks, vs = cache
    return gdn.gdn_attention_paged(q, k, v, table, lens, k_scale=ks, v_scale=vs, scale=scale, cu_seqlens=cu, o=o,
                                   workspace=workspace)


def check_attention(o, q, cache, table, lens, cu, scale, label):
    """o against the oracle: the weights are rounded to bf16 in the products and in their sum (2 x 2^-8 of the same sum
    over |v|), the result once (2^-8 of it); scores are exact products with 2^-24 for each of 128 additions: 2^-17 of
    |q||k| scale, at most 2^-9 here (|q||k| about 128, scale up to 2)."""
    B, T, H, d = q.shape
    sc = 1 / d ** 0.5 if scale is None else scale
    ref, a = paged.attention(f64(q).reshape(-1, H, d), values(cache[0], cache[2]), values(cache[1], cache[3]), f64(table).astype(int),
                             f64(lens).astype(int), None if cu is None else f64(cu).astype(int), B, T, sc)
    got = f64(o).reshape(-1, H, d)
    rows = ~np.isnan(a).any((1, 2))
    assert np.isfinite(got[rows]).all(), label
    off = np.abs(got - ref)[rows] / np.maximum((3 * 2.0 ** -8 + 2.0 ** -9) * a[rows], 1e-30)
    print("  %s: largest error %.3f of the bound" % (label, off.max() if off.size else 0), flush=True)
    assert (off <= 1).all(), label
    return rows
