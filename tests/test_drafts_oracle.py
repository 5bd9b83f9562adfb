"""Pins of the oracle of a drafted step (``oracle/drafts.py``), CPU."""
from fractions import Fraction

import numpy as np
import pytest

import oracle
from oracle import drafts


def test_tables_by_hand():
    """Sequence 0 shrinks from 3 pages to 1, sequence 1 grows from 1 to 3, sequence 2 keeps a shared page at length 0."""
    table = [[5, 2, 7, -1], [0, -1, -1, -1], [9, 4, -1, -1]]
    t, held, free, n_free, missing = drafts.cache_tables([10, 40, 0], table, [3, 1, 2], [1, 3, 6, 8, -1, -1, -1, -1, -1, -1], 4, 16, [0, 0, 1])
    assert t.tolist() == [[5, -1, -1, -1], [0, 7, 4, -1], [9, -1, -1, -1]]      # pool 1 3 6 8 | 2 7 4: the last two
    assert held.tolist() == [1, 3, 1] and n_free == 5 and missing == 0
    assert free.tolist() == [1, 3, 6, 8, 2, 7, 4, -1, -1, -1]
    # and back: the pool as before
    t, held, free, n_free, missing = drafts.cache_tables([48, 10, 30], t, held, free, n_free, 16, [0, 0, 1])
    assert n_free == 4 and held.tolist() == [3, 1, 2] and free[:4].tolist() == [1, 3, 6, 8]
    assert sorted(t[0, :3].tolist() + t[2, 1:2].tolist()) == [2, 4, 5, 7]


def test_tables_short_pool():
    t, held, free, n_free, missing = drafts.cache_tables([40, 33], [[-1] * 3, [-1] * 3], [0, 0], [4, 2, 0, 1], 4, 16)
    assert t.tolist() == [[4, 2, 0], [1, -1, -1]] and held.tolist() == [3, 1] and (n_free, missing) == (0, 2)


@pytest.mark.parametrize("seed", range(5))
def test_pages_are_conserved(seed):
    r = np.random.default_rng(seed)
    n, width, n_pages, page = 7, 9, 40, 16
    table, held, free, n_free = np.full((n, width), -1), np.zeros(n, dtype=int), r.permutation(n_pages), n_pages
    for _ in range(40):
        table, held, free, n_free, missing = drafts.cache_tables(r.integers(0, 170, n), table, held, free, n_free, page)
        mine = [int(table[i, e]) for i in range(n) for e in range(held[i])]
        assert sorted(mine + free[:n_free].tolist()) == list(range(n_pages))
        assert all((table[i, held[i]:] == -1).all() for i in range(n)) and (missing == 0 or n_free == 0)


def test_maps_by_hand():
    cu, pos, slots = drafts.step_maps([18, 2, 40], [[3, 1], [0, -1], [2, 9]], 5, 16, 9, [3, 4, 1])
    assert cu.tolist() == [0, 3, 7, 8]
    assert pos.tolist() == [15, 16, 17, -2, -1, 0, 1, 39, 0]
    assert slots.tolist() == [63, 16, 17, -1, -1, 0, 1, -1, -1]


def test_draft_step_is_decode_steps():
    r = np.random.default_rng(1)
    q, k, v = (r.standard_normal(s) for s in ((2, 5, 1, 4), (2, 5, 1, 4), (2, 5, 2, 3)))
    g, beta, S = r.standard_normal((2, 5, 2)), r.standard_normal((2, 5, 2)), r.standard_normal((2, 2, 3, 4))
    kw = dict(qk_l2norm=True, gate_logits=True)
    o, S_new = drafts.draft_step(q, k, v, g, beta, S, [3, 0], **kw)
    state = S
    for t in range(5):
        y, state = oracle.decode_step_ex(q[:, t], k[:, t], v[:, t], g[:, t], beta[:, t], state, **kw)
        assert np.allclose(y, o[:, t], rtol=1e-13, atol=1e-13)
        if t == 2:
            assert np.allclose(S_new[0], state[0], rtol=1e-13, atol=1e-13)
    assert (S_new[1] == S[1]).all()


def test_verify_by_hand():
    p = np.array([[[.5, .25, .25, 0], [0, .5, 0, .5], [.25] * 4]])
    q = np.array([[[.25, .5, .25, 0], [.5, .5, 0, 0]]])
    run = lambda x, u, lens=None: [y.tolist() for y in drafts.verify(p, q, [x], lens, [u])]   # noqa: E731
    assert run([0, 1], [.999, .999, 0.]) == [[[0, 1, 0]], [3]]         # p >= q: taken; the lowest of the last row
    assert run([0, 1], [.999, .999, .75]) == [[[0, 1, 3]], [3]]        # 3/4 of the last row: the border is the next one's
    assert run([1, 1], [.5, 0, .5]) == [[[0, -1, -1]], [1]]            # 1/2 q = p: not taken; p - q is positive at 0 alone
    assert run([1, 1], [.4999, .9999, .5]) == [[[1, 1, 2]], [3]]
    assert run([0, 0], [0, 0, .9]) == [[[0, 3, -1]], [2]]              # p = 0 of the second
    assert run([0, 1], [0, 0, .3], [1]) == [[[0, 1, -1]], [2]]         # one draft: behind it from row 1 (0, 1/2, 0, 1/2)
    assert run([0, 7], [0, 0, .9]) == [[[0, 3, -1]], [2]]              # outside the vocabulary
    assert [y.tolist() for y in drafts.verify(p, None, [[0, 1]], None, [[.49, .5, .1]])] == [[[0, 3, -1]], [2]]
    assert [y.tolist() for y in drafts.verify(np.zeros((1, 1, 3)), None, None, None, [[.2]])] == [[[-1]], [1]]


def test_verified_tokens_are_distributed_as_the_target():
    """Over drafts drawn from q and all u: P(first token = x) = q(x) min(1, p/q) + P(no draft taken) w(x) / W = p(x)."""
    p, q = [Fraction(a, 16) for a in (1, 8, 4, 3, 0)], [Fraction(a, 16) for a in (4, 4, 4, 2, 2)]
    taken = [b * min(Fraction(1), a / b) for a, b in zip(p, q)]
    w = [max(a - b, Fraction(0)) for a, b in zip(p, q)]
    assert [t + (1 - sum(taken)) * x / sum(w) for t, x in zip(taken, w)] == p
    # ... and the oracle takes and draws just so, over a grid of 64 values of each u
    rows = np.array([[[float(a) for a in p], [1, 0, 0, 0, 0]]])
    count = [Fraction(0)] * 5
    for x in range(5):
        for a in range(64):
            for b in range(64):
                t, c = drafts.verify(rows, np.array([[[float(y) for y in q]]]), [[x]], None, [[a / 64, b / 64]])
                count[t[0, 0]] += q[x] / 64 ** 2
    assert max(abs(float(c - a)) for c, a in zip(count, p)) < 2 / 64   # (either draw of 64 misses a border by under 1/64)
