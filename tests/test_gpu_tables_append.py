"""What gdn_cache_tables says of a step's rows is what the entry points that take its tables do: gdn_kv_append writes a token at its
slot and nowhere else, turned by its position."""
import numpy as np
import pytest
import torch

import paged_cases as pc
import paper_2607_14568_amd as gdn
from paged_cases import normal

pytestmark = pytest.mark.gpu
i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32).cuda()   # noqa: E731


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("short", [0, 3])
@pytest.mark.parametrize("dense", [False, True])
def test_slots_are_where_tokens_go(dense, short, page):
    """``short``: pages that the pool lacks, so that the last sequences' tokens have no slot."""
    print("case: slots", dense, short, page, flush=True)
    r = np.random.default_rng(page + short)
    n, Hkv, d = 9, 2, 64
    new = np.full(n, 4) if dense else r.integers(0, 2 * page, n)
    lens = new + r.integers(0, 5 * page, n)
    need = -(-lens // page)
    n_pages, width = int(need.sum()) - short, int(need.max()) + 1
    T = int(new.sum()) + (0 if dense else 5)
    shape = (n, 4) if dense else (1, T)
    table, held = i32(np.full((n, width), -1)), i32(np.zeros(n))
    pos, slots = torch.full((T,), 9, dtype=torch.int32).cuda(), torch.full((T,), 9).cuda()
    cu, missing = i32(np.zeros(n + 1)), i32([0])
    gdn.gdn_cache_tables(i32(lens), table, held, i32(r.permutation(n_pages)), i32([n_pages]), page, missing=missing, cu_seqlens=cu,
                         new_lens=None if dense else i32(new), positions=pos, slots=slots)
    assert missing.item() == short
    k, v = normal(1, *shape, Hkv, d).cuda(), normal(2, *shape, Hkv, d).cuda()
    cache = [torch.full((n_pages, Hkv, page, d), 7.0, dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    f = pc.freqs(d).cuda()
    gdn.gdn_kv_append(k, v, *cache, table, i32(lens), inv_freq=f, cu_seqlens=None if dense else cu)
    _, turned = gdn.gdn_qk_norm_rope(k, k, inv_freq=f, positions=pos.view(shape).contiguous())
    there = slots >= 0
    at = slots[there]
    assert there[:int(new.sum())].any() and (short > 0) == bool((~there[:int(new.sum())]).any()) and not there[int(new.sum()):].any()
    assert len(set(at.tolist())) == at.numel()
    for c, x in zip(cache, (turned, v)):
        rows = c.transpose(1, 2).reshape(-1, Hkv, d)
        want = x.reshape(T, Hkv, d)[there].float()
        # (the same products in fp32, rounded to bf16 once: a step of it apart at most)
        assert ((rows[at].float() - want).abs() <= 2.0 ** -7 * want.abs() + 2.0 ** -18).all()
        assert torch.equal(rows[at].float(), want) or x is turned
        left = torch.ones(rows.shape[0], dtype=torch.bool, device="cuda")
        left[at] = False
        assert (rows[left] == 7).all()
