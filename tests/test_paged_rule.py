"""The rule that cuts a step of gdn_attention_paged into items: no lengths make more of them than the grid has, and no two
parts share one (CPU)."""
import random

import pytest

import paged_rule as rule
import paper_2607_14568_amd as gdn


def _step(rng):
    """Sizes of a call, and new tokens and lengths of its sequences."""
    H = rng.choice([1, 2, 6, 8, 16, 24, 32, 64])
    Hkv = rng.choice([h for h in (1, 2, 3, 4, 6, 8, 16, 64) if H % h == 0 and h <= H])
    page, packed = rng.choice([16, 32, 64, 128]), rng.random() < 0.5
    n = rng.choice([1, 2, 3, 7, 30, 64, 65, 130, 300])
    longest = rng.choice([100, 777, 3000, 20000, 140000, 2000000])
    if packed:
        new = [rng.choice([0, 1, 1, 1, 2, 5, rng.randrange(1, 400)]) for _ in range(n)]
        T = max(1, sum(new)) + rng.choice([0, 0, 9])
        B = 1
    else:
        T, B = rng.choice([1, 1, 1, 2, 4, 17, 100, 2048]), n
        new = [T] * n
    kind = rng.choice(["alike", "uniform", "one long", "logs"])
    lens = {"alike": lambda: longest, "uniform": lambda: rng.randrange(longest + 1), "one long": lambda: rng.randrange(100),
            "logs": lambda: int(longest ** rng.random())}[kind]
    lens = [m + lens() for m in new]
    if kind == "one long":
        lens[rng.randrange(n)] = longest
    if rng.random() < 0.1:
        lens[rng.randrange(n)] = rng.choice([0, -5, 2 ** 31 - 1])
    max_pages = -(-max(max(lens) if max(lens) < 2 ** 30 else longest, 1) // page) * rng.choice([1, 1, 2, 10]) + rng.choice([0, 1])
    return B, T, H, Hkv, page, max_pages, n if packed else 0, new, lens


@pytest.mark.parametrize("seed", range(8))
def test_items_fit_their_grid(seed):
    rng = random.Random(seed)
    grown = fell = cut = 0
    for _ in range(400):
        B, T, H, Hkv, page, max_pages, n_seqs, new, lens = _step(rng)
        p = rule.plan(B, T, H, Hkv, page, max_pages, n_seqs)
        assert gdn.gdn_attention_paged_workspace_bytes(B, T, H, Hkv, 128, page, max_pages, n_seqs) == rule.workspace(p, Hkv, 128)
        parts, count = rule.items(p, new, lens)
        case = (B, T, H, Hkv, page, max_pages, n_seqs, new, lens)
        assert count <= p["items"], case
        assert len(set(parts)) == len(parts) and all(0 <= w < count for w in parts), case
        _, g, f, _ = rule.cut(p, new, lens)
        grown, fell, cut = grown + (g > 0), fell + f, cut + (len(parts) > sum(-(-m * p["G"] // p["rb"]) for m in new))
    print("grown %d, fell back %d, cut %d of 400" % (grown, fell, cut))
    assert grown > 10 and fell > 10 and cut > 100   # (all branches, many times over the seeds)


def test_the_largest_sums():
    """Lengths whose units reach 2^23 a sequence, over as many sequences as are ever cut, all in one lane of the sum."""
    rng = random.Random(3)
    for _ in range(30):
        n = rng.choice([500, 2000, 40000])
        lens, new = [0] * n, [0] * n
        for i in range(0, n, 64):
            lens[i], new[i] = rng.randrange(1, 2 ** 30), 1
        T = sum(new)
        p = rule.plan(1, T, 2, 1, 128, 2 ** 23, n)
        parts, count = rule.items(p, new, lens)
        assert p["spare"] > 0 and count <= p["items"] and len(set(parts)) == len(parts)
