"""The bounds of tests/draft_bounds.py tell a wrong recurrence from a right one, at every length that the GPU tests take (CPU)."""
import numpy as np
import pytest

import draft_bounds as db
from oracle import drafts

f64 = lambda t: t.double().numpy()   # noqa: E731
SIZES = [(1, 1, 1), (2, 5, 2), (3, 8, 2), (2, 9, 1), (1, 16, 1), (1, 35, 2)]   # B, T, key heads of 2


@pytest.mark.parametrize("raw", [False, True])
@pytest.mark.parametrize("B,T,Hk", SIZES)
def test_the_tiles_are_the_recurrence(B, T, Hk, raw):
    x = [f64(y) for y in db.make(T, (B, T), B, 2, Hk, 64, 64, "f32", raw)]
    keep = [T - 1] * B
    o, S, off_o, off_S = db.walk(*x, keep, None, raw, 0.5)
    ro, rS = drafts.draft_step(*x, keep=keep, qk_l2norm=raw, gate_logits=raw, scale=0.5)
    assert np.abs(o - ro).max() < 1e-12 and np.abs(S - rS).max() < 1e-12


def fp32(x, keep, raw, scale):
    """Token by token in fp32, products summed one after another: within the bounds as well."""
    f = np.float32
    q, k, v, g, beta, S = (y.astype(f) for y in x)
    if raw:
        q, k = (y / np.sqrt((y * y).sum(-1, keepdims=True, dtype=f) + f(1e-6)) for y in (q, k))
        g, beta = -(np.maximum(g, f(0)) + np.log1p(np.exp(-np.abs(g)))), f(1) / (f(1) + np.exp(-beta))
    H = v.shape[2]
    q, k = (np.repeat(y, H // y.shape[2], 2) for y in (q, k))
    dot = lambda M, y: np.add.accumulate(M * y[..., None, :], -1, dtype=f)[..., -1]   # noqa: E731
    o, kept = np.zeros_like(v), S.copy()
    for t in range(v.shape[1]):
        S = np.exp(g[:, t])[..., None, None] * S
        S = S + (beta[:, t][..., None] * (v[:, t] - dot(S, k[:, t])))[..., None] * k[:, t][..., None, :]
        o[:, t] = dot(S, f(scale) * q[:, t])
        for b in range(v.shape[0]):
            if keep[b] == t + 1:
                kept[b] = S[b]
    return o.astype(np.float64), kept.astype(np.float64)


@pytest.mark.parametrize("raw", [False, True])
@pytest.mark.parametrize("dk,dv", [(128, 128), (64, 128)])
@pytest.mark.parametrize("B,T,Hk", SIZES)
def test_bounds_hold_fp32_and_catch_mistakes(B, T, Hk, dk, dv, raw):
    x = [f64(y) for y in db.make(T, (B, T), B, 2, Hk, dk, dv, "f32", raw)]
    keep = [T] * B
    ref = db.walk(*x, keep, None, raw, 0.5)
    fine = db.worst(*fp32(x, keep, raw, 0.5), ref, "f32")
    print("T %d: fp32 token by token %.3f of the bound" % (T, fine))
    assert fine <= 1
    for wrong in ["beta", "gates", "bf16 inputs"] + ["pairs"] * (T > 1) + ["bf16 between tiles"] * (T > db.TILE):
        o, S, _, _ = db.walk(*x, keep, None, raw, 0.5, wrong)
        state, out = db.worst(None, S, ref, "f32"), db.worst(o, ref[1], ref, "f32")
        print("  %s: state %.1f, outputs %.1f of the bound" % (wrong, state, out))
        # (a tile's gates may leave nothing of a mistake before it)
        assert out > 1 and (state > 1 or wrong == "bf16 between tiles"), wrong
