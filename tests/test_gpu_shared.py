"""GPU parity of gdn_attention_shared: the fp64 oracle of attention over a table (``oracle/paged.py``), which knows no prefix,
on tables whose groups' sequences name the same pages."""
import numpy as np
import pytest
import torch

import paged_cases as pc
import paper_2607_14568_amd as gdn
from paged_cases import cuda, normal

pytestmark = pytest.mark.gpu
i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32)   # noqa: E731


def batch(groups, page, seed, extra=3, width=1):
    """``groups``: a list of (prefix tokens, [(own tokens, new tokens), ..]); own None: a sequence without any token (its row of
    the table holds -1); own below 0: one that ends that far inside the prefix.  Returns table, lens, new, prefix, cu_groups, n_pages."""
    need, rows, lens, new = 0, [], [], []
    for prefix, seqs in groups:
        common = list(range(need, need + prefix // page))
        need += len(common)
        for own, m in seqs:
            L = 0 if own is None else max(prefix + own, 0) + m
            pages = -(-L // page)
            mine = common[:pages]
            mine += list(range(need, need + pages - len(mine)))
            need = max([need] + [x + 1 for x in mine])
            rows.append(mine)
            lens.append(L)
            new.append(m)
    n_pages = need + extra
    order = np.random.default_rng(seed).permutation(n_pages)
    table = np.full((len(rows), max(len(r) for r in rows) + width), -1, dtype=np.int32)
    for s, r in enumerate(rows):
        table[s, :len(r)] = order[r]
    cu = np.cumsum([0] + [len(s) for _, s in groups])
    return table, lens, new, [p for p, _ in groups], cu, n_pages


def call(q, cache, table, lens, prefix, cu_groups=None, cu=None, **kw):
    k, v, ks, vs = cache
    return gdn.gdn_attention_shared(q, k, v, table, lens, prefix, cu_groups=cu_groups, k_scale=ks, v_scale=vs, cu_seqlens=cu, **kw)


def run(groups, H, Hkv, d, page, cache, seed, dense=False, scale=None, pad=5, change=None):
    table, lens, new, prefix, cg, n_pages = batch(groups, page, seed)
    kv = pc.make_cache(n_pages, Hkv, page, d, cache, seed)
    n, T = len(new), sum(new)
    q = normal(seed + 9, n, new[0], H, d) if dense else normal(seed + 9, 1, T + pad, H, d)
    cu = None if dense else np.cumsum([0] + new)
    if change:
        change(q, kv, table, lens)
    o = torch.full_like(q, 7.0).cuda()
    one = len(groups) == 1 and seed % 2
    args = cuda(q, i32(table), i32(lens), i32(prefix), None if one else i32(cg), None if dense else i32(cu))
    got = call(args[0], cuda(*kv), args[1], args[2], args[3], args[4], args[5], o=o, scale=scale)
    assert got is o
    if not dense:
        assert (o[0, T:] == 7).all()
        o, q = o[:, :T], q[:, :T]
    label = "%d groups, %d sequences, prefix %s" % (len(groups), n, prefix[:3])
    pc.check_attention(o, q, kv, torch.from_numpy(table), i32(lens), None if dense else i32(cu), scale, label)
    return o


HEADS = [(1, 1, 128), (6, 2, 64), (16, 8, 128), (32, 2, 128), (8, 8, 64), (48, 1, 64)]


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("page", [16, 64, 128])
@pytest.mark.parametrize("H,Hkv,d", HEADS)
def test_one_token_each(H, Hkv, d, page, cache):
    print("case: shared", H, Hkv, d, page, cache, flush=True)
    r = np.random.default_rng(page + d)
    for prefix, n in ((0, 3), (1, 2), (page, 4), (500, 1), (500, 40), (2111, 9)):
        run([(prefix, [(int(a), 1) for a in r.integers(0, 300, n)])], H, Hkv, d, page, cache, prefix + n, dense=True, scale=0.2)


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("page", [16, 32, 128])
@pytest.mark.parametrize("H,Hkv,d", HEADS[:4])
def test_groups_of_uneven_drafts(H, Hkv, d, page, cache):
    """Groups of one and of many, without a prefix, shorter and empty sequences among them (a first one, too), several tokens."""
    print("case: shared groups", H, Hkv, d, page, cache, flush=True)
    r = np.random.default_rng(page)
    seqs = lambda n: [(int(a), int(m)) for a, m in zip(r.integers(0, 400, n), r.integers(0, 7, n))]   # noqa: E731
    run([(700, seqs(5)), (0, seqs(2)), (1300, [(None, 2), (-200, 3)] + seqs(7)), (64, seqs(1))], H, Hkv, d, page, cache, 4)
    run([(900, seqs(4) + [(None, 1)])], H, Hkv, d, page, cache, 5)
    run([(333, [(-400, 2), (None, 1)]), (257, [(0, 1), (0, 2)])], H, Hkv, d, page, cache, 6)


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("H,Hkv,d", [(16, 8, 128), (16, 2, 64)])
def test_pieces_behind_a_prefix(H, Hkv, d, cache):
    """Long pieces of prompts behind it: blocks of 128 rows on both sides of the prefix's end."""
    run([(640, [(100, 200), (0, 77), (1, 1), (500, 300)])], H, Hkv, d, 32, cache, 1)
    run([(640, [(30, 65)] * 3)], H, Hkv, d, 64, cache, 2, dense=True)


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_many_chunks(cache):
    """More chunks than the join takes in one go, on either side of the prefix's end."""
    run([(20000, [(0, 1), (5, 1)])], 2, 1, 128, 64, cache, 1, dense=True)
    run([(64, [(20000, 1), (10, 1)])], 2, 1, 128, 64, cache, 2, dense=True)
    run([(9000, [(3000, 1)] * 9)], 16, 1, 64, 16, cache, 3, dense=True)


@pytest.mark.parametrize("n", [70, 400])
def test_many_sequences(n):
    r = np.random.default_rng(n)
    groups = [(int(p), [(int(a), 1) for a in r.integers(0, 90, n // 10)]) for p in r.integers(0, 400, 10)]
    run(groups, 4, 2, 64, 16, "bf16", n, dense=True)
    run([(50, [(3, 1)] * 2)] * (n // 2), 4, 2, 64, 16, "bf16", n + 1, dense=True)


def test_missing_pages_and_odd_groups():
    """Pages that are not there, inside the prefix and behind it; group offsets outside the contract, sequences behind the last
    group, prefixes below 0 and past the table."""
    table, lens, new, prefix, cg, n_pages = batch([(200, [(50, 1), (90, 1), (10, 1)]), (96, [(40, 1), (1, 1)])], 16, 3)
    table[:3, 4] = -1
    table[:3, 7] = n_pages + 5
    table[1, 13] = -1
    kv = pc.make_cache(n_pages, 2, 16, 128, "bf16", 3)
    q = normal(4, 5, 1, 4, 128)
    for pre, cut in (([200, 96], [0, 3, 5]), ([200, 96], [0, 3, 99]), ([200, 96], [7, 3, 2]), ([200], [0, 2]), ([-5, 96], [0, 3, 5]),
                     ([10 ** 6, 96], [0, 3, 5]), ([200, 2 ** 31 - 1], [0, -2, 0])):
        args = cuda(q, i32(table), i32(lens), i32(pre), i32(cut))
        o = call(args[0], cuda(*kv), *args[1:])
        pc.check_attention(o, q, kv, torch.from_numpy(table), i32(lens), None, None, "%s %s" % (pre, cut))


def test_rows_without_a_key_are_zero():
    o = run([(64, [(None, 3), (5, 2)])], 4, 2, 128, 16, "bf16", 2)
    assert (o[0, :3] == 0).all()
    table = np.full((2, 4), -1, dtype=np.int32)
    kv = pc.make_cache(2, 2, 16, 128, "bf16", 1)
    q = normal(1, 2, 1, 4, 128)
    o = call(*cuda(q), cuda(*kv), *cuda(i32(table), i32([40, 50]), i32([32])))
    assert (o == 0).all()


@pytest.mark.parametrize("n", [2, 40])
@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_what_lies_behind_a_length_is_not_read(cache, n):
    """Slots behind the sequences' lengths hold NaN; the rest of the prefix's last started page is a sequence's own."""
    table, lens, new, prefix, cg, n_pages = batch([(200, [(i, 1) for i in range(n)])], 64, 3)
    kv = pc.make_cache(n_pages, 2, 64, 128, cache, 3)
    for s, L in enumerate(lens):
        for t in range(L, table.shape[1] * 64):
            if table[s, t // 64] >= 0:
                kv[0][table[s, t // 64], :, t % 64] = kv[1][table[s, t // 64], :, t % 64] = float("nan")
    q = normal(5, n, 1, 16, 128)
    args = cuda(q, i32(table), i32(lens), i32(prefix))
    o = call(args[0], cuda(*kv), *args[1:])
    assert torch.isfinite(o).all()


@pytest.mark.parametrize("n", [3, 70])
def test_special_values_of_a_prefix(n):
    """An infinite value of the prefix reaches its channel in every row of the group, a NaN likewise, and no other group's."""
    table, lens, new, prefix, cg, n_pages = batch([(128, [(20, 1)] * n), (128, [(20, 1)] * n)], 64, 3)
    kv = pc.make_cache(n_pages, 1, 64, 64, "bf16", 3)
    kv[1][table[0, 0], 0, 7, 5] = float("inf")
    kv[1][table[0, 1], 0, 9, 6] = float("nan")
    q = normal(5, 2 * n, 1, 2, 64)
    args = cuda(q, i32(table), i32(lens), i32(prefix), i32(cg))
    o = call(args[0], cuda(*kv), *args[1:]).float().cpu()
    assert (o[:n, ..., 5] == float("inf")).all() and torch.isnan(o[:n, ..., 6]).all()
    o[:n, ..., 5:7] = 0
    assert torch.isfinite(o).all()


def test_as_paged():
    """Equal to gdn_attention_paged but for roundings: 2 x 2^-8 of weights, the output's 2^-8."""
    table, lens, new, prefix, cg, n_pages = batch([(3000, [(100 * i, 1) for i in range(30)])], 64, 3)
    kv = cuda(*pc.make_cache(n_pages, 8, 64, 128, "bf16", 3))
    q, t, L = cuda(normal(4, 30, 1, 16, 128), i32(table), i32(lens))
    a, b = call(q, kv, t, L, i32(prefix).cuda()).float(), pc.attend(q, kv, t, L).float()
    assert (a - b).abs().max() < 4 * 2.0 ** -8 * b.abs().max()


def test_captured_and_replayed_with_other_lengths():
    """Lengths, tables, prefixes and groups are read on the device: one graph, three steps, eager calls between."""
    H, Hkv, d, page, n = 8, 2, 128, 32, 12
    sets = []
    for i, p in enumerate(((700, 90), (64, 1500), (0, 33))):
        cuts = [5 + i, n - 5 - i]
        groups = [(p[0], [(40 * j, 1) for j in range(cuts[0])]), (p[1], [(7 * j, 1) for j in range(cuts[1])])]
        table, lens, new, prefix, cg, n_pages = batch(groups, page, i)
        full = np.full((n, 80), -1, dtype=np.int32)
        full[:, :table.shape[1]] = table
        sets.append(cuda(normal(i, n, 1, H, d), i32(full), i32(lens), i32(prefix), i32(cg)))
    kv = cuda(*pc.make_cache(600, Hkv, page, d, "bf16", 3))
    ws = [torch.empty(gdn.gdn_attention_shared_workspace_bytes(n, 1, H, Hkv, d, page, 80, 0, 2), dtype=torch.uint8, device="cuda") for _ in "ab"]
    want = [call(s[0], kv, *s[1:], workspace=ws[0]) for s in sets]
    x, o = [t.clone() for t in sets[0]], torch.empty_like(sets[0][0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(x[0], kv, *x[1:], o=o, workspace=ws[1])
    for i in (0, 1, 2, 1, 0):
        for a, b in zip(x, sets[i]):
            a.copy_(b)
        o.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, want[i]), i
        assert torch.equal(call(sets[0][0], kv, *sets[0][1:], workspace=ws[0]), want[0])


def test_streams():
    """Calls on streams of their own at once, a workspace each."""
    table, lens, new, prefix, cg, n_pages = batch([(2000, [(30 * i, 1) for i in range(20)])], 64, 3)
    kv = cuda(*pc.make_cache(n_pages, 4, 64, 128, "e4m3", 3))
    t, L, p = cuda(i32(table), i32(lens), i32(prefix))
    qs = [normal(i, 20, 1, 16, 128).cuda() for i in range(3)]
    want = [call(q, kv, t, L, p) for q in qs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in qs]
    got = [[] for _ in qs]
    for _ in range(5):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[i].append(call(qs[i], kv, t, L, p))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want[i]) for i, g in enumerate(got) for o in g)
