"""Pins of the oracle of the attention layers' serving operators (``oracle/paged.py``), CPU."""
import math

import numpy as np
import pytest
import torch

from oracle import attention as att
from oracle import paged

rng = np.random.default_rng


def test_norm_and_rotation_by_hand():
    x = [3.0, -4.0, 1.0, 2.0]
    r = 1 / math.sqrt((9 + 16 + 1 + 4) / 4 + 0.5)
    got = paged.norm(np.array(x), np.array([1.0, 2.0, 0.5, -1.0]), 0.5)
    assert np.allclose(got, [3 * r, -8 * r, 0.5 * r, -2 * r], rtol=1e-15)
    f, p = [0.7, 0.01], 11
    y = np.array(x + [5.0])[None, None]
    c, s = [math.cos(p * t) for t in f], [math.sin(p * t) for t in f]
    half = [3 * c[0] - 1 * s[0], -4 * c[1] - 2 * s[1], 1 * c[0] + 3 * s[0], 2 * c[1] - 4 * s[1], 5]
    near = [3 * c[0] + 4 * s[0], -4 * c[0] + 3 * s[0], 1 * c[1] - 2 * s[1], 2 * c[1] + 1 * s[1], 5]
    assert np.allclose(paged.rotate(y, [p], f)[0, 0], half, rtol=1e-14)
    assert np.allclose(paged.rotate(y, [p], f, True)[0, 0], near, rtol=1e-14)


@pytest.mark.parametrize("near", [False, True])
def test_rotated_products_depend_on_the_distance(near):
    q, k = rng(1).standard_normal((2, 1, 1, 16))
    f = 10000.0 ** (-np.arange(6) / 6)
    at = [(q_at, k_at) for q_at, k_at in [(5, 2), (1003, 1000), (100003, 100000)]]
    dots = [(paged.rotate(q, [i], f, near) * paged.rotate(k, [j], f, near)).sum() for i, j in at]
    assert np.allclose(dots, dots[0], atol=1e-9) and abs(dots[0] - (q * k).sum()) > 1e-3


def test_e4m3_is_torchs_rounding():
    y = np.concatenate([rng(2).uniform(-448, 448, 4000), 10.0 ** rng(3).uniform(-4, 2.6, 4000), [0, 448, 2 ** -10, 3 * 2.0 ** -10]])
    want = torch.from_numpy(y).to(torch.float8_e4m3fn).double().numpy()
    assert (paged.e4m3(y) == want).all()


@pytest.mark.parametrize("amax,want", [(448.0, 1.0), (448.0001, 2.0), (1.75, 2.0 ** -8), (1.76, 2.0 ** -7), (0.0, 2.0 ** -100)])
def test_power_scale(amax, want):
    assert paged.power_scale(amax) == want


def test_appending_in_steps():
    """A prompt in one call and in steps fills the same cells; an 8-bit page's scale grows with its tokens."""
    rows = rng(4).standard_normal((40, 2, 8)) * np.linspace(0.1, 30, 40)[:, None, None]
    table = np.array([[2, 0, 3, -1]])
    once, step = np.zeros((4, 2, 16, 8)), np.zeros((4, 2, 16, 8))
    paged.append(once, None, table, [40], rows, None, 1, 40, 16)
    for a, b in [(0, 1), (1, 20), (20, 40)]:
        paged.append(step, None, table, [b], rows[a:b], None, 1, b - a, 16)
    assert (once == step).all() and (once[2, :, 5] == rows[5]).all() and (once[3, :, 7] == rows[39]).all() and not once[1].any()
    codes, scale = np.zeros((4, 2, 16, 8)), np.zeros((4, 2))
    for t in range(40):
        paged.append(codes, scale, table, [t + 1], rows[t:t + 1], None, 1, 1, 16)
    for b, lo in ((2, 0), (0, 16), (3, 32)):
        part = rows[lo:lo + 16]
        assert (scale[b] == [paged.power_scale(np.abs(part[:, h]).max()) for h in range(2)]).all()
        back = codes[b].transpose(1, 0, 2)[:len(part)] * scale[b][:, None]
        assert (np.abs(back - part) <= 2.0 ** -4 * np.abs(part) + 2.0 ** -9 * scale[b][:, None]).all()


def test_attention_is_the_prompts_attention():
    """A prompt's queries over its own cache: causal attention; the last ones alone: its last rows."""
    T, H, Hkv, d = 37, 4, 2, 8
    q, k, v = (rng(5 + i).standard_normal((T, h, d)) for i, h in enumerate((H, Hkv, Hkv)))
    table = np.array([[1, 3, 0]])
    kc, vc = np.full((2, 4, Hkv, 16, d), 9e9)
    paged.append(kc, None, table, [T], k, None, 1, T, 16)
    paged.append(vc, None, table, [T], v, None, 1, T, 16)
    want = att.causal_attention(q[None], k[None], v[None], 0.3)[0]
    o, a = paged.attention(q, kc, vc, table, [T], None, 1, T, 0.3)
    assert np.allclose(o, want, atol=1e-12) and (a >= np.abs(o) - 1e-12).all()
    assert np.allclose(paged.attention(q[-5:], kc, vc, table, [T], None, 1, 5, 0.3)[0], want[-5:], atol=1e-12)
    # a missing page leaves its keys out; no key at all: zeros
    gone, _ = paged.attention(q[-1:], kc, vc, np.array([[1, -1, 0]]), [T], None, 1, 1, 0.3)
    keep = np.r_[0:16, 32:37]
    assert np.allclose(gone[0], att.causal_attention(np.repeat(q[None, -1:], 21, 1), k[None, keep], v[None, keep], 0.3)[0, -1])
    assert not paged.attention(q[:2], kc, vc, table, [1], None, 1, 2, 0.3)[0][0].any()


def test_packed_offsets_are_clamped():
    assert paged.spans(1, 10, [0, 4, 4, 10]) == [(0, 4), (4, 0), (4, 6)]
    assert paged.spans(1, 10, [0, 7, 3, 99, -2]) == [(0, 7), (7, 0), (7, 3), (10, 0)]
