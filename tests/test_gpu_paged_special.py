"""Values that are not finite in a paged cache: what rows that see them, and rows that do not, make of them."""
import numpy as np
import pytest
import torch

import paged_cases as pc
from oracle import paged
from paged_cases import cuda, f64, normal

pytestmark = pytest.mark.gpu
# new tokens a sequence: blocks of 16 rows (1, 4), of 128 (100: 4 sequences x 13 blocks of 16 rows x 2 heads are too many)
NEW = [1, 4, 100]


def _case(cache, new, page, d, seed):
    n, H, Hkv = 4, 4, 2
    lens = [new + 190, new + 70, new + 64, new + 3]
    q = normal(seed, n, new, H, d)
    table, n_pages = pc.pages_for(lens, page, seed)
    return q, list(pc.make_cache(n_pages, Hkv, page, d, cache, seed)), table, lens


def _at(table, page, s, p):
    return int(table[s, p // page]), p % page


def _check(q, kc, table, lens, label):
    """Element by element as the oracle has it: NaN where it is NaN, the same infinity, else within check_attention's bound
    (3.5 x 2^-8 of the sum over |v|)."""
    n, new, H, d = q.shape
    with np.errstate(invalid="ignore"):
        ref, a = paged.attention(f64(q).reshape(-1, H, d), pc.values(kc[0], kc[2]), pc.values(kc[1], kc[3]), table, lens, None, n, new,
                                 d ** -0.5)
    got = f64(pc.attend(q.cuda(), cuda(*kc), torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32).cuda())).reshape(ref.shape)
    for kind, of in (("NaN", np.isnan), ("+inf", np.isposinf), ("-inf", np.isneginf)):
        print("  %s: %s %d of %d" % (label, kind, of(got).sum(), of(ref).sum()), flush=True)
    assert (np.isnan(got) == np.isnan(ref)).all() and (np.isposinf(got) == np.isposinf(ref)).all()
    assert (np.isneginf(got) == np.isneginf(ref)).all()
    fine = np.isfinite(ref)
    assert (np.abs(got[fine] - ref[fine]) <= (3 * 2.0 ** -8 + 2.0 ** -9) * a[fine] + 1e-30).all()
    return ref


@pytest.mark.parametrize("page,d", [(16, 128), (64, 64), (128, 128)])
@pytest.mark.parametrize("new", NEW)
def test_infinite_values(new, page, d):
    """An infinity makes its channel that infinity in every row that sees it, two opposite ones NaN, a NaN NaN: at keys that all
    rows of the call see, and at keys among the new tokens, which some see."""
    print("case: infinite values", new, page, d, flush=True)
    q, kc, table, lens = _case("bf16", new, page, d, page + new)
    inf = float("inf")
    mid = new // 2
    for s, h, p, c, x in [(0, 0, 5, 3, -inf), (0, 0, 190 + mid, 7, inf), (0, 1, 190 + mid, 0, -inf), (1, 0, 70, 9, inf),
                          (1, 0, 70 + mid, 9, -inf), (1, 0, 70 + mid, 11, -inf), (2, 1, 64 + mid, 2, float("nan")), (2, 1, 64 + mid, 4, inf),
                          (3, 0, 3 + new - 1, d - 1, inf), (3, 1, 0, d - 2, -inf)]:
        i, slot = _at(table, page, s, p)
        kc[1][i, h, slot, c] = x
    ref = _check(q, kc, table, lens, "infinite values")
    assert np.isposinf(ref).any() and np.isneginf(ref).any() and np.isnan(ref).any()


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("new", NEW)
def test_scales_that_are_no_numbers(new, page):
    """A NaN as the scale of a page of values, or of keys, under codes that are numbers: rows that see one of the page's keys are
    NaN in every channel, all others as without it."""
    print("case: NaN scales", new, page, flush=True)
    q, kc, table, lens = _case("e4m3", new, page, 128, 30 + page)
    for s, h, p, i in [(0, 0, lens[0] - 1, 3), (1, 1, lens[1] - new // 2 - 1, 3), (2, 0, lens[2] - 1, 2), (3, 1, 0, 3)]:
        kc[i][_at(table, page, s, p)[0], h] = float("nan")
    ref = _check(q, kc, table, lens, "NaN scales")
    assert np.isnan(ref).any() and np.isfinite(ref).any()


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("new", NEW)
def test_negative_scales_and_zero(new, page):
    """A scale of either sign, powers of two and others, and 0: a code stands for its product with it."""
    print("case: negative scales", new, page, flush=True)
    q, kc, table, lens = _case("e4m3", new, page, 128, 40 + page)
    g = np.random.default_rng(page)
    for i in (2, 3):
        kc[i] *= torch.from_numpy(g.choice([1.0, -1.0, -1.25, 0.0], tuple(kc[i].shape))).float()
    _check(q, kc, table, lens, "negative scales")
