"""gdn_draft_verify at the ends of its ranges over rows of many slices: whole numbers, equal to what the definition gives."""
import numpy as np
import pytest
import torch

import paper_2607_14568_amd as gdn
from paged_cases import f64

pytestmark = pytest.mark.gpu
IO = {"bf16": torch.bfloat16, "f32": torch.float32}


def rows(seed, n, V, io, spread=12.0):
    """Probabilities [n, V] of a wide spread, in double and rounded to ``io``."""
    x = spread * np.random.default_rng(seed).standard_normal((n, V))
    x = np.exp(x - x.max(-1, keepdims=True))
    return torch.from_numpy(x / x.sum(-1, keepdims=True)).to(IO[io])


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("V", [900, 5000, 9001, 70001])
@pytest.mark.parametrize("u", [1.0, 1.5, float("inf")])
def test_one_or_more_draws_the_last_token(u, V, io):
    """The last token that has any probability, however little, and whatever the order of the sums rounds to."""
    n = 40
    p = rows(V, n, V, io)
    ends = V - 1 - np.arange(n) % 7
    for s in range(n):
        p[s, ends[s]:] = 0
        p[s, ends[s]] = 1e-25
    t, c = gdn.gdn_draft_verify(p[:, None].contiguous().cuda(), torch.full((n, 1), u).cuda())
    assert (c == 1).all() and t[:, 0].tolist() == ends.tolist()
    # behind a draft that is refused, from what is left of p: the same token, which the draft's own row lacks
    q = rows(V + 1, n, V, io)[:, None].contiguous()
    x = q[:, 0].argmax(-1, keepdim=True).int()
    for s in range(n):
        p[s, x[s, 0]] = 0
        q[s, 0, ends[s]:] = 0
    us = torch.tensor([[0.5, u]]).repeat(n, 1)
    t, c = gdn.gdn_draft_verify(torch.stack([p, p], 1).cuda(), us.cuda(), drafts=x.cuda(), q=q.cuda())
    assert (c == 1).all() and t[:, 0].tolist() == ends.tolist() and (t[:, 1] == -1).all()


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("n,V", [(1, 1000), (37, 20001)])
def test_a_step_without_drafts(n, V, io):
    """m = 0 with a serving loop's buffers: lengths, whatever they hold, drafts and their rows of no token."""
    p, u = rows(V, n, V, io, 2.0)[:, None].contiguous(), torch.rand(n, 1, generator=torch.Generator().manual_seed(n))
    sums = np.cumsum(f64(p)[:, 0].astype(np.longdouble), -1)
    goal = f64(u)[:, 0].astype(np.longdouble) * sums[:, -1]
    assert (np.abs(sums - goal[:, None]).min(-1) > 2.0 ** -40).all()   # (no draw on a border)
    want = [int(np.searchsorted(a, b, side="right")) for a, b in zip(sums, goal)]
    p, u = p.cuda(), u.cuda()
    none, lens = torch.empty(n, 0, dtype=torch.int32, device="cuda"), torch.arange(n, dtype=torch.int32, device="cuda") - 3
    empty = torch.empty(n, 0, V, dtype=IO[io], device="cuda")
    for kw in ({}, dict(draft_lens=lens), dict(drafts=none), dict(drafts=none, q=empty, draft_lens=lens)):
        t, c = gdn.gdn_draft_verify(p, u, **kw)
        assert t[:, 0].tolist() == want and (c == 1).all()
    for kw in (dict(draft_lens=lens[:0]), dict(drafts=lens[:, None]), dict(q=p), dict(draft_lens=lens.long())):
        with pytest.raises((ValueError, TypeError)):
            gdn.gdn_draft_verify(p, u, **kw)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("V", [300, 5001, 70001, 200003])
def test_nothing_left_of_the_target(V, io):
    """q equal to p and a draft that u = 1 refuses: no max(p - q, 0) is positive, and the token is drawn from p by all its slices; the
    same for a certain draft on a row that holds nothing else."""
    n = 5
    p = rows(V, n, V, io, 2.0)
    u = torch.rand(n, 2, generator=torch.Generator().manual_seed(V))
    u[:, 0] = 1.0
    sums = np.cumsum(f64(p).astype(np.longdouble), -1)
    goal = f64(u)[:, 1].astype(np.longdouble) * sums[:, -1]
    assert (np.abs(sums - goal[:, None]).min(-1) > 2.0 ** -40).all()   # (no draw on a border)
    want = [int(np.searchsorted(a, b, side="right")) for a, b in zip(sums, goal)]
    x = p.argmax(-1, keepdim=True).int()
    both = torch.stack([p, p.flip(-1)], 1).cuda()
    for _ in range(3):
        t, c = gdn.gdn_draft_verify(both, u.cuda(), drafts=x.cuda(), q=both[:, :1].contiguous())
        assert t[:, 0].tolist() == want and (c == 1).all() and (t[:, 1] == -1).all()
    one = torch.zeros(n, 2, V, dtype=IO[io])
    at = [0, V - 1, V // 2, 299, 7]
    for s in range(n):
        one[s, 0, at[s]] = 1.0
    t, c = gdn.gdn_draft_verify(one.cuda(), u.cuda(), drafts=torch.tensor(at, dtype=torch.int32)[:, None].cuda())
    assert t[:, 0].tolist() == at and (c == 1).all()
