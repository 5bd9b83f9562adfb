"""Weights of gdn_attention_shared, whichever blocks its rows go in: held in more bits than bf16 has."""
import numpy as np
import pytest
import torch

import paged_cases as pc
from oracle import paged
from paged_cases import cuda, f64, normal
from test_gpu_shared import batch, call, i32

pytestmark = pytest.mark.gpu

# (d, H, H_kv, groups): rows of a prefix in blocks of 16, in blocks of 128 with own keys by 16, and both in blocks of 128
CASES = [(128, 4, 2, [(256, [(30, 1), (77, 1), (1, 1)])]),
         (128, 4, 2, [(256, [(3 * i, 1) for i in range(24)])]),
         (64, 6, 2, [(192, [(3 * i, 1) for i in range(30)]), (320, [(5, 1)] * 30)]),
         (128, 8, 1, [(256, [(5 * i, 4) for i in range(9)])]),
         (128, 4, 1, [(192, [(40, 70), (0, 90), (100, 33)])]),
         (64, 2, 2, [(256, [(0, 100), (20, 100)])])]


def make(cache, n_pages, Hkv, page, d, factor=1.0):
    """Keys of about unit size and values of +-1, in the cache's type; 8-bit scales are ``factor`` times a power of two."""
    k, v, ks, vs = pc.make_cache(n_pages, Hkv, page, d, cache, 5)
    signs = torch.from_numpy(np.random.default_rng(7).choice([-1.0, 1.0], v.shape))
    if ks is None:
        return k, signs.to(v.dtype), None, None
    codes = torch.from_numpy(np.clip(f64(k.float()) / 8, -448, 448)).to(torch.float8_e4m3fn)
    return codes, (signs * 64).to(v.dtype), torch.full_like(ks, 0.125) * factor, torch.full_like(vs, 2.0 ** -6) * factor


def check(cache, d, H, Hkv, groups, page, factor=1.0):
    table, lens, new, prefix, cg, n_pages = batch(groups, page, 3)
    dense = len(set(new)) == 1
    n, T = len(new), sum(new)
    shape = (n, new[0]) if dense else (1, T)
    q = (normal(d + H, *shape, H, d, dtype=torch.float32) / 8).bfloat16()
    cu = None if dense else np.cumsum([0] + new)
    kc = make(cache, n_pages, Hkv, page, d, factor)
    most = np.linalg.norm(f64(q), axis=-1).max() * np.linalg.norm(pc.values(kc[0], kc[2]), axis=-1).max()
    assert most * d ** -0.5 <= 25 * 128 ** -0.5 and max(lens) <= 380
    ref, a = paged.attention(f64(q).reshape(-1, H, d), pc.values(kc[0], kc[2]), pc.values(kc[1], kc[3]), table, lens, cu, *shape, d ** -0.5)
    o = call(q.cuda(), cuda(*kc), *cuda(i32(table), i32(lens), i32(prefix), i32(cg)), None if dense else i32(cu).cuda())
    off = np.abs(f64(o).reshape(ref.shape) - ref) / (2.0 ** -8 * np.abs(ref) + 2.0 ** -13 * a)
    print("  largest error %.3f of the bound" % off.max(), flush=True)
    assert (off <= 1).all()


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("d,H,Hkv,groups", CASES)
def test_weights_keep_more_than_bf16(d, H, Hkv, groups, page, cache):
    """Values of +-1 under weights of about the same size, whose sums nearly cancel, so that roundings of single weights show.

    Bound, beside the result's own rounding (2^-8 of it), relative to a, the sum of weight |v|:
      weights   two bf16 numbers: 2^-15, and 2^-20
      scores    d <= 128 exact products summed in fp32: 2^-17 |q||k| scale, |q||k| <= 25 for queries of size 1/8, scale 128^-1/2:
                2^-15.8 of a weight, in the sum over v and in that of the weights: 2^-14.8
      sums      up to 380 additions in fp32, both sums, joined by up to 20 more: 2 * 400 * 2^-24 = 2^-14.4
    together under 2^-13.  (Weights rounded to bf16 are off by 2^-8 / 3^1/2 on average, outputs of 300 keys by about 2^-13.4 on
    average, and by several times that among these thousands.)"""
    print("case: shared weights", cache, page, d, H, Hkv, flush=True)
    check(cache, d, H, Hkv, groups, page)


@pytest.mark.parametrize("n,new", [(4, 1), (24, 1), (3, 70)])
def test_an_infinite_value_of_little_weight(n, new):
    """An infinity in the prefix under a weight of 2^-92 of the others': its channel is that infinity in every row of either block
    size, and no other channel is."""
    table, lens, _, prefix, cg, n_pages = batch([(192, [(40, new)] * n)], 64, 3)
    k, v = (torch.zeros(n_pages, 1, 64, 64, dtype=torch.bfloat16) for _ in "kv")
    q = torch.zeros(n, new, 2, 64, dtype=torch.bfloat16)
    q[..., 0] = 8
    k[table[0, 1], 0, 9, 0] = -64                        # (8 * 64 / 64^1/2 = 64 = 92.3 log 2)
    v[table[0, 1], 0, 9, 5] = float("inf")
    v[table[0, 1], 0, 9, 6] = -float("inf")
    o = call(q.cuda(), cuda(k, v, None, None), *cuda(i32(table), i32(lens), i32(prefix))).float().cpu()
    assert (o[..., 5] == float("inf")).all() and (o[..., 6] == -float("inf")).all()
    o[..., 5:7] = 0
    assert (o == 0).all()
