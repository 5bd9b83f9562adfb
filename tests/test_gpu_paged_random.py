"""Steps of random sizes: appended, then attended, each held to the fp64 oracle."""
import random

import pytest
import torch

import paged_cases as pc
from paged_cases import cuda, f64
from test_gpu_paged import _append, _append_case, _check_append

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("seed", range(16))
def test_a_random_step(cache, seed):
    rng = random.Random(seed)
    Hkv = rng.choice([1, 2, 3, 5, 8])
    H, d, page = Hkv * rng.choice([1, 2, 3, 7]), rng.choice([64, 128]), rng.choice([16, 32, 64, 128])
    n, packed = rng.choice([1, 2, 5, 9, 66]), rng.random() < 0.5
    most = rng.choice([1, 4, 40, 150]) if n < 20 else rng.choice([1, 3])
    new = [rng.randrange(most + 1) for _ in range(n)] if packed else [rng.randrange(1, most + 1)] * n
    new[0] = max(new[0], 1)
    lens = [m + int(rng.choice([10, 300, 1500]) * rng.random()) for m in new]
    rot, near, width = rng.choice([0, 16, d // 2, d]), rng.random() < 0.5, rng.choice([1, 40])
    cu = [sum(new[:i]) for i in range(n + 1)] if packed else None
    T = cu[-1] + rng.choice([0, 7]) if packed else None
    print("case: random", cache, seed, H, Hkv, d, page, n, packed, new[:8], lens[:8], rot, near, flush=True)
    c = _append_case(cache, page, d, H, Hkv, lens, new, cu, rot, near, seed, T=T)
    if width > 1:
        table = torch.full((n, c["table"].shape[1] + width), -1, dtype=torch.int32).numpy()
        table[:, :c["table"].shape[1]] = c["table"]
        c["table"] = table
    qt, dev = _append(c)
    _check_append(c, qt, dev, "append")
    kc = [dev[0], dev[1], dev[2], dev[3]]
    at = torch.tensor(lens, dtype=torch.int32).cuda()
    tab, cut = torch.from_numpy(c["table"]).cuda(), None if cu is None else torch.tensor(cu, dtype=torch.int32).cuda()
    q = torch.where(torch.isfinite(qt), qt, qt.new_zeros(()))
    o = torch.full_like(q, 7.0)
    pc.attend(q, kc, tab, at, cut, None, o)
    rows = pc.check_attention(o, q, kc, tab, at, cut, None, "attention")
    assert (f64(o).reshape(-1, H, d)[~rows] == 7.0).all()
