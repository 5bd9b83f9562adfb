"""Weights of gdn_attention_paged where rows go in blocks of 16: held in more bits than bf16 has."""
import numpy as np
import pytest
import torch

import paged_cases as pc
from oracle import paged
from paged_cases import cuda, f64, normal

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("d,H,Hkv,new,lens,max_pages", [
    (128, 4, 2, 1, [300, 77, 1, 33], 5), (64, 6, 2, 1, [300, 64], 5), (128, 4, 1, 4, [200, 31, 4, 100], 4),
    (128, 2, 1, 1, [400], 2000)])
def test_weights_keep_more_than_bf16(cache, d, H, Hkv, new, lens, max_pages):
    """Values of +-1 under weights of about the same size, whose sums nearly cancel, so that roundings of single weights show.

    Bound, beside the result's own rounding (2^-8 of it), relative to a = sum of weight |v| = 1:
      weights   two bf16 numbers: 2^-15, and 2^-20
      scores    d <= 128 exact products summed in fp32: 2^-17 |q||k| scale, |q||k| <= 25 for queries of size 1/8, scale 128^-1/2:
                2^-15.8 of a weight, in the sum over v and in that of the weights: 2^-14.8
      sums      400 additions in fp32, both sums: 2 * 400 * 2^-24 = 2^-14.4
    together under 2^-13.  (Weights rounded to bf16 are off by 2^-8 / 3^1/2 on average, outputs of 300 keys by about 2^-13.4 on
    average, and by several times that among these thousands.)"""
    print("case: weights", cache, d, H, Hkv, new, lens, max_pages, flush=True)
    n, page = len(lens), 64
    q = (normal(d + H, n, new, H, d, dtype=torch.float32) / 8).bfloat16()
    table, n_pages = pc.pages_for(lens, page, 3)
    table = np.pad(table, ((0, 0), (0, max(0, max_pages - table.shape[1]))), constant_values=-1)
    k, v, ks, vs = pc.make_cache(n_pages, Hkv, page, d, cache, 5)
    if ks is not None:
        k, ks = (f64(k.float()) / 64), torch.full_like(ks, 0.125)
        k = torch.from_numpy(np.clip(k * 8, -448, 448)).to(torch.float8_e4m3fn)
    signs = torch.from_numpy(np.random.default_rng(7).choice([-1.0, 1.0], v.shape))
    v = signs.to(v.dtype) if vs is None else (signs * 64).to(v.dtype)
    vs = None if vs is None else torch.full_like(vs, 2.0 ** -6)
    kc = (k, v, ks, vs)
    most = np.linalg.norm(f64(q), axis=-1).max() * np.linalg.norm(pc.values(k, ks), axis=-1).max()
    assert most * d ** -0.5 <= 25 * 128 ** -0.5
    ref, a = paged.attention(f64(q).reshape(-1, H, d), pc.values(k, ks), pc.values(v, vs), table, lens, None, n, new, d ** -0.5)
    assert np.allclose(a, 1)
    o = pc.attend(q.cuda(), cuda(*kc), torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32).cuda())
    off = np.abs(f64(o).reshape(ref.shape) - ref) / (2.0 ** -8 * np.abs(ref) + 2.0 ** -13)
    print("  largest error %.3f of the bound" % off.max(), flush=True)
    assert (off <= 1).all()
