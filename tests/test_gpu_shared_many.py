"""gdn_attention_shared with more than 64 sequences, whose parts one workgroup works out ahead: packed and dense, many groups, blocks
of either size on both sides of the prefix's end, offsets outside the contract."""
import numpy as np
import pytest
import torch

import paged_cases as pc
from paged_cases import cuda, normal
from test_gpu_shared import batch, call, i32, run

pytestmark = pytest.mark.gpu


def drafts(r, n, top, most=6):
    return [(int(a), int(m)) for a, m in zip(r.integers(0, top, n), r.integers(0, most + 1, n))]


@pytest.mark.parametrize("H,Hkv,d,page,cache", [(4, 2, 128, 16, "bf16"), (4, 2, 128, 64, "e4m3"), (8, 1, 64, 32, "e4m3"), (6, 2, 64, 128, "bf16")])
@pytest.mark.parametrize("n", [65, 300, 600])
def test_packed_drafts(n, H, Hkv, d, page, cache):
    """0 to 6 new tokens each (every tenth sequence without any), sequences that end inside the prefix, rows behind the last one."""
    print("case: shared many packed", n, H, Hkv, d, page, cache, flush=True)
    r = np.random.default_rng(n + d)
    cut = n // 3
    run([(400, drafts(r, cut, 90)), (0, drafts(r, 5, 300)), (250, [(-100, 2), (None, 3)] + drafts(r, n - cut - 7, 200))], H, Hkv, d, page, cache, n)
    run([(320, drafts(r, n, 60))], H, Hkv, d, page, cache, 2 * n + 1)


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("n", [70, 300])
def test_dense_at_128(n, cache):
    r = np.random.default_rng(n)
    groups = [(int(p), [(int(a), 2) for a in r.integers(0, 150, n // 5)]) for p in r.integers(0, 500, 5)]
    run(groups, 8, 2, 128, 32, cache, n, dense=True)


@pytest.mark.parametrize("size", [1, 2])
def test_more_groups_than_threads(size):
    """300 and 520 groups of two sequences and one, some without a prefix, some without a token."""
    r = np.random.default_rng(size)
    many = [(int(p), drafts(r, size, 60, 2)) for p in r.integers(0, 200, 520 if size == 1 else 300)]
    run(many, 4, 2, 64, 16, "bf16", 2 + size)


@pytest.mark.parametrize("cache,d", [("bf16", 128), ("e4m3", 128), ("e4m3", 64)])
def test_many_rows_a_sequence(cache, d):
    """Blocks of 128 rows on both sides: more than 64 rows a sequence on average."""
    print("case: shared many rows", cache, d, flush=True)
    r = np.random.default_rng(d)
    run([(200, [(int(a), int(m)) for a, m in zip(r.integers(0, 80, 66), r.integers(0, 25, 66))])], 16, 2, d, 32, cache, 4)
    run([(130, [(9, 10)] * 40), (300, [(50, 10)] * 30)], 16, 2, d, 64, cache, 6, dense=True)


def test_as_many_sequences_as_a_call_takes():
    r = np.random.default_rng(1)
    run([(96, [(int(a), 1) for a in r.integers(0, 40, 1500)]), (64, [(int(a), 1) for a in r.integers(0, 40, 548)])], 2, 1, 64, 16, "bf16", 2, dense=True)


def test_offsets_outside_the_contract():
    """Token offsets that fall back, lie below 0 and pass the rows; group offsets likewise: clamped to a partition."""
    n, page = 80, 16
    groups = [(160, [(int(i % 30), 2) for i in range(50)]), (96, [(5, 2)] * 30)]
    table, lens, new, prefix, cg, n_pages = batch(groups, page, 3)
    kv = pc.make_cache(n_pages, 2, page, 64, "bf16", 3)
    T = 2 * n
    q = normal(4, 1, T, 4, 64)
    even = list(range(0, T + 1, 2))
    lows, highs = list(even), list(even)
    lows[5], lows[60] = -7, 3                       # below 0, below the one ahead of it: empty sequences, the next ones longer
    highs[70:] = [T + 50] * (n + 1 - 70)            # the 70th sequence takes the rest
    for cu in (even, lows, highs):
        for pre, cut in ((prefix, cg), (prefix, [9, 50, 999]), (prefix, [0, 50, 20]), ([160, 0, 96], [0, 50, 40, 2 ** 31 - 1])):
            print("case: shared offsets", cu is lows, cu is highs, list(cut), flush=True)
            args = cuda(q, i32(table), i32(lens), i32(pre), i32(cut), i32(cu))
            o = call(args[0], cuda(*kv), *args[1:])
            pc.check_attention(o, q, kv, torch.from_numpy(table), i32(lens), i32(cu), None, "%s" % list(cut))
