"""gdn_draft_step within the roundings of its fp32 steps (``draft_bounds.py``, whose bounds a wrong recurrence misses by far): every
size of head, one tile of tokens and several, packed sequences, every way to keep tokens."""
import numpy as np
import pytest
import torch

import draft_bounds as db
import paper_2607_14568_amd as gdn
from oracle import drafts
from paged_cases import f64

pytestmark = pytest.mark.gpu
i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32).cuda()   # noqa: E731


def check(x, keep, cu, raw, scale, io, label):
    """Outputs and state of one call, the state of one without outputs, against the oracle's values and the counted bounds."""
    flags = gdn.GDN_QK_L2NORM | gdn.GDN_GATE_LOGITS if raw else 0
    args = [f64(y) for y in x]
    ref = db.walk(*args, keep, cu, raw, scale)
    o, S = drafts.draft_step(*args, keep=keep, cu=cu, qk_l2norm=raw, gate_logits=raw, scale=scale)
    assert np.nanmax(np.abs(o - ref[0])) < 1e-11 and np.abs(S - ref[1]).max() < 1e-11
    ref = (o, S) + ref[2:]
    d = [y.cuda() for y in x]
    kw = dict(keep=None if keep is None else i32(keep), cu_seqlens=None if cu is None else i32(cu), flags=flags)
    S1, S2 = d[5].clone(), d[5].clone()
    got = gdn.gdn_draft_step(*d[:5], S1, scale=scale, **kw)
    assert gdn.gdn_draft_step(None, *d[1:5], S2, **kw) is None
    off = db.worst(f64(got), f64(S1), ref, io), db.worst(None, f64(S2), ref, io)
    print("  %s: %.4f and %.4f of the bound" % (label, *off), flush=True)
    assert max(off) <= 1, label


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("dk,dv", [(128, 128), (64, 64), (128, 64), (64, 128)])
@pytest.mark.parametrize("B,T,H,Hk", [(1, 1, 2, 1), (2, 5, 6, 2), (3, 8, 2, 2), (2, 9, 4, 1), (1, 16, 2, 1), (1, 35, 2, 2), (17, 3, 8, 8)])
def test_dense(B, T, H, Hk, dk, dv, io):
    print("case: draft exact", B, T, H, Hk, dk, dv, io, flush=True)
    for raw in (False, True):
        x = db.make(B + T, (B, T), B, H, Hk, dk, dv, io, raw)
        some = np.random.default_rng(T).integers(0, T + 1, B)
        for keep in (None, [0] * B, some, [max(T - 1, 1)] * B, [min(9, T)] * B):
            check(x, keep, None, raw, 0.5, io, "raw %d keep %s" % (raw, None if keep is None else list(keep)[:4]))


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("dk,dv", [(128, 128), (64, 128)])
def test_packed(dk, dv, io):
    """No token, one, several tiles; rows behind the last sequence; more sequences than a wave has lanes."""
    print("case: draft exact packed", dk, dv, io, flush=True)
    for raw, lens in ((False, [3, 0, 17, 9, 1, 8]), (True, list(np.random.default_rng(3).integers(0, 20, 150)))):
        cu = [0] + list(np.cumsum(lens))
        n = len(lens)
        x = db.make(n, (1, cu[-1] + 4), n, 4, 2, dk, dv, io, raw)
        for keep in (None, [int(z) for z in np.random.default_rng(n).integers(0, np.array(lens) + 1)]):
            check(x, keep, cu, raw, 1.0, io, "%d sequences raw %d keep %s" % (n, raw, keep is not None))
