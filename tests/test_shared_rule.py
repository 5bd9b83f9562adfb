"""The rule that cuts a step of gdn_attention_shared into items, written out on the host after its comments in gdn.hip and
shared.hip: no lengths make more of them than the grid and the workspace have, and no two parts share one (CPU)."""
import random

import pytest

import paper_2607_14568_amd as gdn

UNIT, CUS = 128, 256
up = lambda a, b: -(-a // b)   # noqa: E731


def plan(B, T, H, Hkv, page, max_pages, n_seqs, groups):
    G, n = H // Hkv, n_seqs or B
    tokens = B * T
    rows, units = tokens * G, up(page * max_pages, UNIT)
    p = dict(round=max(1, 2 * CUS // Hkv), rbp=16 if rows <= 32 * groups else 128, rbt=16 if rows <= 64 * n else 128, G=G)
    blocks_p = rows // p["rbp"] + min(groups, tokens)
    p["blocks_t"] = rows // p["rbt"] + min(n, tokens) if n_seqs else B * up(T * G, p["rbt"])
    p["items_p"] = min(blocks_p + p["round"], blocks_p * units)
    p["items_t"] = min(p["blocks_t"] + p["round"], p["blocks_t"] * units)
    return p


def workspace(p, n, groups, Hkv, d):
    at = lambda size: up(size, 256) * 256   # noqa: E731
    rows = [p["items_p"] * Hkv * p["rbp"], p["items_t"] * Hkv * p["rbt"]]
    small = [n * 16, groups * 16, n * 48, (groups + 1) * 4, (n + 1) * 4, (n + 1) * 4, 4]
    return sum(map(at, small)) + sum(at(r * 8) + at(r * d * 4) for r in rows)


def parts(p, new, lens, prefix, ends, cap, page):
    """(rows, keys, start) of every group's prefix and of every sequence."""
    groups, seqs, at = [], [], 0
    for g, end in enumerate(ends):
        P = min(max(prefix[g], 0), cap) // page * page
        shares = [P > 0 and new[s] > 0 and max(lens[s], 0) - new[s] >= P for s in range(at, end)]
        groups.append((sum(new[at:end]) * p["G"] if any(shares) else 0, P))
        seqs += [(new[s] * p["G"], max(lens[s], 0), P if x else 0) for s, x in zip(range(at, end), shares)]
        at = end
    seqs += [(new[s] * p["G"], max(lens[s], 0), 0) for s in range(at, len(new))]
    return groups, seqs


def items(p, groups, seqs, cap):
    """Numbers of the groups' items and of the sequences' that have work."""
    rb = [(up(r, p["rbp"]), up(P, UNIT)) for r, P in groups]
    rt = [(up(r, p["rbt"]), max(up(min(L, cap) - a, UNIT), 1)) for r, L, a in seqs]
    c = max(min(up(sum(b * u for b, u in rb + rt), p["round"]), 1 << 23), 1)

    def numbers(blocks, keys_of):
        out, first = [], 0
        for i, (nb, u) in enumerate(blocks):
            for b in range(nb):
                keys, chunks = keys_of(i, b), 1
                if keys > c * UNIT:
                    chunks = up(keys, c * UNIT)
                    size = up(up(keys, chunks), UNIT) * UNIT
                    chunks = up(keys, size)
                out += [first + j * nb + (b if j % 2 else nb - 1 - b) for j in range(chunks)]
            first += nb * up(u, c)
        return out, first

    def own(s, b):
        rows, L, a = seqs[s]
        m = rows // p["G"]
        return min(max(L - m + min((b * p["rbt"] + p["rbt"] - 1) // p["G"], m - 1) + 1, 0), cap) - a
    return numbers(rb, lambda g, b: groups[g][1]), numbers(rt, own)


def _step(rng):
    H = rng.choice([1, 2, 6, 8, 16, 24, 32, 64])
    Hkv = rng.choice([h for h in (1, 2, 3, 4, 6, 8, 16, 64) if H % h == 0 and h <= H])
    page, packed, n = rng.choice([16, 32, 64, 128]), rng.random() < 0.5, rng.choice([1, 2, 3, 7, 30, 64, 65, 130, 300])
    new = [rng.choice([0, 1, 1, 1, 2, 5, rng.randrange(1, 200)]) for _ in range(n)] if packed else [rng.choice([1, 1, 2, 4, 17, 100])] * n
    if not sum(new):
        new[0] = 1
    groups = rng.choice([1, 1, min(n, 4), n])
    ends = sorted(rng.randrange(n + 1) for _ in range(groups - 1)) + [rng.choice([n, n, rng.randrange(n + 1)])]
    ends = [max(ends[:i + 1]) for i in range(groups)]
    prefix = [int(rng.choice([200, 3000, 70000, 2000000]) ** rng.random()) for _ in range(groups)]
    top, lens, at = rng.choice([0, 10, 500, 5000]), [], 0
    for g, e in enumerate(ends + [n]):
        lens += [new[s] + (prefix[g] if g < groups else 0) + int(top * rng.random() ** 2) for s in range(at, e)]
        at = e
    if rng.random() < 0.2:
        lens[rng.randrange(n)] = rng.choice([0, -5, 2 ** 31 - 1])
    max_pages = up(max([x for x in lens if x < 2 ** 30] + [1]), page) + rng.choice([0, 1, 50])
    B, T = (1, sum(new) + rng.choice([0, 0, 9])) if packed else (n, new[0])
    return B, T, H, Hkv, page, max_pages, n if packed else 0, groups, new, lens, prefix, ends


@pytest.mark.parametrize("seed", range(6))
def test_items_fit_their_grid(seed):
    rng = random.Random(seed)
    cut = shared = 0
    for _ in range(300):
        B, T, H, Hkv, page, max_pages, n_seqs, groups, new, lens, prefix, ends = _step(rng)
        p = plan(B, T, H, Hkv, page, max_pages, n_seqs, groups)
        assert gdn.gdn_attention_shared_workspace_bytes(B, T, H, Hkv, 128, page, max_pages, n_seqs, groups) == workspace(p, len(new), groups, Hkv, 128)
        cap = page * max_pages
        g, s = parts(p, new, lens, prefix, ends, cap, page)
        case = (B, T, H, Hkv, page, max_pages, n_seqs, groups, new, lens, prefix, ends)
        for (used, count), most in zip(items(p, g, s, cap), (p["items_p"], p["items_t"])):
            assert count <= most, case
            assert len(set(used)) == len(used) and all(0 <= w < count for w in used), case
        assert sum(up(r, p["rbt"]) for r, _, _ in s) <= p["blocks_t"], case
        cut, shared = cut + (items(p, g, s, cap)[0][1] > 1), shared + any(r for r, _ in g)
    print("prefixes cut %d, shared %d of 300" % (cut, shared))
    assert cut > 50 and shared > 100
