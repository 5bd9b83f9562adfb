"""gdn_attention_paged over every way its rule cuts a step into items, against the fp64 oracle; page and head sizes that the
cases of test_gpu_paged.py leave out."""
import numpy as np
import pytest
import torch

import paged_cases as pc
import paged_rule as rule
from paged_cases import cuda, f64, normal

pytestmark = pytest.mark.gpu


def _lens(seed, n, most):
    return [int(x) for x in np.random.default_rng(seed).integers(1, most, n)]


def _run(label, cache, H, Hkv, d, page, new, lens, packed=False, spare_rows=0, width=1):
    """The call against the oracle; returns the rule's plan, (units per chunk, growth steps, fell back) and the parts it made."""
    print("case: cuts", label, cache, H, Hkv, d, page, new[:6], lens[:6], flush=True)
    n = len(lens)
    B, T = (1, sum(new) + spare_rows) if packed else (n, new[0])
    table, n_pages = pc.pages_for(lens, page, n, width=width)
    q, kc = normal(n + d, B, T, H, d), pc.make_cache(n_pages, Hkv, page, d, cache, n)
    cu = [0] + [int(x) for x in np.cumsum(new)] if packed else None
    cu = None if cu is None else torch.tensor(cu, dtype=torch.int32).cuda()
    dev, at = cuda(*kc), torch.tensor(lens, dtype=torch.int32).cuda()
    tab = torch.from_numpy(table).cuda()
    p = rule.plan(B, T, H, Hkv, page, table.shape[1], n if packed else 0)
    o = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    pc.attend(q.cuda(), dev, tab, at, cu, None, o)
    rows = pc.check_attention(o, q, kc, tab, at, cu, None, label)
    assert (f64(o).reshape(-1, H, d)[~rows] == 7.0).all()
    return p, rule.cut(p, new, lens)[:3], len(rule.items(p, new, lens)[0])


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("H,d,page", [(16, 128, 64), (32, 64, 16)])
def test_chunks_grow_until_they_fit(cache, H, d, page):
    """Blocks of 16 rows: the first size gives too many items, a larger one fits (one long sequence among short ones)."""
    p, (c, grown, fell), parts = _run("grow", cache, H, 16, d, page, [1] * 6, [40000, 50, 300, 900, 1500, 20])
    assert p["rb"] == 16 and grown > 0 and not fell and parts > p["blocks"]


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("kind", ["even lengths", "packed"])
def test_chunks_by_the_spare_items(cache, kind):
    """Blocks of 16 rows: lengths for which no size leaves the chip evenly loaded; chunks by the items that the grid has to spare."""
    if kind == "packed":
        new = [int(x) for x in np.random.default_rng(5).integers(0, 3, 70)]
        lens = [m + int(4000 ** x) for m, x in zip(new, np.random.default_rng(6).random(70))]
        p, (c, grown, fell), parts = _run(kind, cache, 12, 12, 64, 16, new, lens, packed=True, spare_rows=3)
        blocks = sum(m > 0 for m in new)
    else:
        p, (c, grown, fell), parts = _run(kind, cache, 8, 8, 128, 64, [1] * 64, [100 * (i + 1) for i in range(64)])
        blocks = 64
    assert p["rb"] == 16 and grown > 0 and fell and parts > blocks


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_uneven_lengths_and_more_blocks_than_items_at_once(cache):
    """30 sequences of 32 heads, more than are resident at once: every size fails, so that the spare items decide."""
    p, (c, grown, fell), parts = _run("not at once", cache, 32, 32, 64, 64, [1] * 30, _lens(30, 30, 5000))
    assert p["rb"] == 16 and p["round"] < 30 and fell and parts > 30


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("H,Hkv", [(24, 12), (9, 3), (6, 6)])
def test_head_counts_that_are_no_powers_of_two(cache, H, Hkv):
    p, _, parts = _run("heads", cache, H, Hkv, 128, 32, [4] * 7, [3000, 2500, 2000, 3100, 700, 1000, 100])
    assert p["rb"] == 16 and parts > p["blocks"]


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("d,page", [(64, 64), (64, 128), (128, 16), (128, 128)])
def test_packed_pieces_in_several_chunks(cache, d, page):
    """Blocks of 128 rows, packed, with an empty sequence and rows behind the last; cut into several chunks each."""
    p, _, parts = _run("packed pieces", cache, 6, 3, d, page, [150, 0, 3, 90, 1], [2150, 10, 900, 1200, 700], packed=True, spare_rows=9)
    assert p["rb"] == 128 and parts > 3 * p["blocks"]


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("d,page", [(64, 128), (128, 32)])
def test_pieces_whose_chunks_grow(cache, d, page):
    """Blocks of 128 rows, more heads: a larger chunk than the first fits."""
    p, (c, grown, fell), parts = _run("pieces grow", cache, 32, 32, d, page, [130] * 3, [1577, 2010, 1232])
    assert p["rb"] == 128 and grown > 0 and not fell and parts > p["blocks"]


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("d,page", [(64, 64), (64, 128), (128, 64)])
def test_pieces_uncut(cache, d, page):
    """Blocks of 128 rows of short sequences: one chunk each, lengths that end inside blocks of keys and pages."""
    p, _, parts = _run("pieces uncut", cache, 10, 5, d, page, [33] * 4, [33, 34, 96, 161])
    assert p["rb"] == 128 and parts == 4


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("new,lens", [(1, [777]), (1, [1]), (3, [300, 5])])
def test_a_table_as_wide_as_the_longest_context(cache, new, lens):
    """Short sequences under a table of 131072 keys: cut and joined, or not, by what they hold."""
    p, _, _ = _run("wide table", cache, 16, 8, 128, 64, [new] * len(lens), lens, width=2048)
    assert p["spare"] > 0


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_pieces_captured_and_on_two_streams(cache):
    """Blocks of 128 rows, cut and joined: a captured call replays with other lengths and queries, eager calls between, bit by bit as
    those; two streams at once with a workspace each do too."""
    H, Hkv, d, page, n, new = 6, 3, 128, 32, 4, 60
    old = [3000, 40, 1000, 0]
    lens = [new + x for x in old]
    print("case: pieces captured", cache, flush=True)
    table, n_pages = pc.pages_for([x + 300 for x in lens], page, 3)
    p = rule.plan(n, new, H, Hkv, page, table.shape[1], 0)
    assert p["rb"] == 128 and p["spare"] > 0 and len(rule.items(p, [new] * n, lens)[0]) > p["blocks"]
    kc, tab = cuda(*pc.make_cache(n_pages, Hkv, page, d, cache, 4)), torch.from_numpy(table).cuda()
    qs = [normal(60 + i, n, new, H, d).cuda() for i in range(3)]
    ats = [torch.tensor([x + 100 * i for x in lens], dtype=torch.int32).cuda() for i in range(3)]
    need = rule.workspace(p, Hkv, d)
    ws = [torch.empty(need, dtype=torch.uint8, device="cuda") for _ in range(3)]
    want = [pc.attend(q, kc, tab, at, workspace=ws[0]) for q, at in zip(qs, ats)]
    q, at, o = qs[0].clone(), ats[0].clone(), torch.empty_like(qs[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pc.attend(q, kc, tab, at, o=o, workspace=ws[1])
    for i in (0, 1, 2, 0):
        q.copy_(qs[i])
        at.copy_(ats[i])
        graph.replay()
        again = pc.attend(qs[i], kc, tab, ats[i], workspace=ws[0])
        torch.cuda.synchronize()
        assert torch.equal(o, want[i]) and torch.equal(again, want[i]), i
    streams, got = [torch.cuda.Stream() for _ in range(3)], []
    for st, x, y, w in zip(streams, qs, ats, ws):
        with torch.cuda.stream(st):
            got.append([pc.attend(x, kc, tab, y, workspace=w) for _ in range(4)])
    torch.cuda.synchronize()
    assert all(torch.equal(x, w) for xs, w in zip(got, want) for x in xs)
