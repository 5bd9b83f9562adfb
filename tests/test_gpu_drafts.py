"""GPU parity of a drafted step's entry points (gdn_cache_tables, gdn_draft_step, gdn_draft_verify) against ``oracle/drafts.py``:
whole numbers equal, states and outputs within bounds counted in roundings."""
import numpy as np
import pytest
import torch

import paper_2607_14568_amd as gdn
from oracle import drafts
from paged_cases import HALF, f64

pytestmark = pytest.mark.gpu
IO = {"bf16": torch.bfloat16, "f32": torch.float32}
i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32).cuda()   # noqa: E731
ints = lambda t: t.cpu().long().numpy()   # noqa: E731


# ------------------------------------------------------------------ gdn_cache_tables
def _pool(n, width, n_pages, seed):
    return np.full((n, width), -1), np.zeros(n, dtype=int), np.random.default_rng(seed).permutation(n_pages), n_pages


def _step(state, lens, page, shared=None, new=None, rows=0, dense=False):
    """One call on the device and in the oracle, everything compared; the state after it."""
    table, held, free, n_free = state
    n = len(lens)
    d = [i32(table), i32(held), i32(free), i32([n_free])]
    missing, cu = i32([77]), i32([-5] * (n + 1)) if new is not None or dense else None
    pos = torch.full((n, rows // n) if dense else (rows,), 55, dtype=torch.int32, device="cuda") if rows else None
    slots = torch.full((n, rows // n) if dense else (rows,), 55, dtype=torch.int64, device="cuda") if rows else None
    gdn.gdn_cache_tables(i32(lens), *d, page, shared=None if shared is None else i32(shared), missing=missing,
                         new_lens=None if new is None else i32(new), cu_seqlens=cu, positions=pos, slots=slots)
    want = drafts.cache_tables(lens, table, held, free, n_free, page, shared)
    got = [ints(x) for x in d]
    assert (got[0] == want[0]).all() and (got[1] == want[1]).all() and got[3][0] == want[3] and ints(missing)[0] == want[4]
    assert (got[2] == want[2]).all()
    if rows:
        wc, wp, ws = drafts.step_maps(lens, want[0], len(free), page, rows, new)
        assert (ints(cu) == wc).all() and (ints(pos).reshape(-1) == wp).all() and (ints(slots).reshape(-1) == ws).all()
    return want[0], want[1], want[2], want[3]


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("n", [1, 2, 7, 64, 65, 300])
def test_tables_steps(n, page):
    """Sequences grow, shrink, end and start again; packed maps with padding, dense ones, none; a pool that runs out."""
    print("case: tables", n, page, flush=True)
    r = np.random.default_rng(n + page)
    state = _pool(n, 12, max(4, n * 5), n)
    for step in range(8):
        lens = r.integers(-3 if step % 3 == 2 else 0, 11 * page, n)
        new = np.minimum(r.integers(0, 9, n), np.maximum(lens, 0) + 1)     # (one position below 0 here and there)
        dense = step % 4 == 3
        state = _step(state, lens, page, None, None if dense or step == 0 else new, n * 3 if dense else 0 if step == 0 else int(new.sum()) + 5,
                      dense)


def test_tables_shared_pages_stay():
    r = np.random.default_rng(5)
    n, page = 9, 16
    table, held, free, n_free = _pool(n, 20, 200, 1)
    table[:, :4] = free[196:]
    table[6:, :4] = -1                                   # (three sequences without the prefix)
    state, shared = (table, np.array([4] * 6 + [0] * 3), free, 196), [4] * 6 + [0] * 3
    for step in range(6):
        lens = r.integers(0, 19 * page, n)
        state = _step(state, lens if step % 2 else lens // 4, page, shared, r.integers(1, 6, n), 60)
        assert (state[0][:6, :4] == state[2][196:]).all() and (state[1][:6] >= 4).all()


def test_tables_take_and_give_back_restores_the_pool():
    state = _pool(40, 30, 700, 3)
    r = np.random.default_rng(4)
    old = r.integers(0, 200, 40)
    state = _step(state, old, 16)
    after = _step(_step(state, old + r.integers(1, 200, 40), 16), old, 16)
    assert all((np.array(a) == np.array(b)).all() for a, b in zip(state[:2], after[:2]))
    assert after[3] == state[3] and (after[2][:after[3]] == state[2][:state[3]]).all()


@pytest.mark.parametrize("n,rows", [(3, 9000), (1100, 3000), (2500, 20000), (4, 8192), (4, 8193), (4, 4096), (4, 4097)])
def test_tables_many(n, rows):
    """Sequences past one round of the workgroup's threads, rows past the launch that takes both."""
    print("case: tables many", n, rows, flush=True)
    r = np.random.default_rng(rows)
    new = r.multinomial(rows - 7, np.ones(n) / n)
    lens = new + r.integers(0, 300, n)
    state = _pool(n, int(lens.max()) // 16 + 2, int((-(-lens // 16)).sum()) - 3, 1)
    state = _step(state, lens, 16, None, new, rows)
    state = _step(state, lens // 2, 16, None, new, rows)
    _step(state, lens, 16, None, None, n * 4, True)


def test_tables_odd_values():
    """Counters and offsets outside the contract: taken as the nearest, more new tokens than rows, lengths past the table."""
    table, held, free, n_free = _pool(4, 5, 30, 2)
    _step((table, held, free, 999), [10, 2000, -7, 33], 16, None, [3, -2, 4, 90], 21)
    _step((table, np.array([9, -3, 0, 5]), free, -4), [80, 80, 0, 80], 16, [9, 1, -1, 0], [1, 1, 1, 1], 4)


# ------------------------------------------------------------------ gdn_draft_step
def _draft_inputs(seed, rows, n, H, Hk, dk, dv, io, raw):
    r = np.random.default_rng(seed)
    t = lambda *s: torch.from_numpy(r.standard_normal(s))   # noqa: E731
    q, k, v, a, b, S = t(*rows, Hk, dk), t(*rows, Hk, dk), t(*rows, H, dv), t(*rows, H), t(*rows, H), 0.3 * t(n, H, dv, dk)
    if not raw:
        q, k = (x / x.norm(dim=-1, keepdim=True) for x in (q, k))
        a, b = -torch.nn.functional.softplus(a - 1), torch.sigmoid(b)
    return [x.to(IO[io]).cuda() for x in (q, k, v)] + [x.float().cuda() for x in (a, b, S)]


def _check_draft(x, o, S, keep, cu, T, io, raw, label, scale=1.0):
    """Unit q and k, gates of 0 to 1: with N the length of a state row plus the sum of the tokens' |v|, no state row gets longer
    than N and no product is over N (1 + scale).  Each of a dot product's 128 fp32 steps and a token's 2 T is off by 2^-24
    of that, and a token's error meets the later ones once each: (128 + 2 T)(T + 1) 2^-24 (N + 1).  bf16 keys and queries are
    what the oracle takes; an output is rounded once."""
    args = [f64(y) for y in x]
    ref_o, ref_S = drafts.draft_step(*args, keep=keep, cu=cu, qk_l2norm=raw, gate_logits=raw, scale=scale)
    H, dv = args[2].shape[2:]
    N = np.sqrt((args[5] ** 2).sum(-1)).max() + np.abs(args[2]).max() * T + 1
    slack = (128 + 2 * T) * (T + 1) * 2.0 ** -24 * N * (1 + scale)
    worst = np.abs(f64(S) - ref_S) / (slack + 2.0 ** -24 * np.abs(ref_S))
    if o is not None:
        live = ~np.isnan(ref_o)
        off = np.abs(f64(o) - ref_o)[live] / (slack + HALF[IO[io]] * np.abs(ref_o[live]))
        worst = np.concatenate([worst.ravel(), off])
    print("  %s: largest error %.3f of the bound" % (label, worst.max()), flush=True)
    assert (worst <= 1).all(), (label, worst.max())


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("dk,dv", [(128, 128), (64, 64), (128, 64), (64, 128)])
@pytest.mark.parametrize("B,T,H,Hk", [(1, 1, 1, 1), (2, 5, 6, 2), (3, 8, 2, 2), (2, 9, 4, 1), (1, 16, 2, 1), (1, 35, 2, 2), (17, 3, 32, 8),
                                      (40, 9, 16, 16)])
def test_draft_step(io, dk, dv, B, T, H, Hk):
    """Few states (a wave each 16 rows) and many (64 rows), one tile of tokens and several, every way to keep them."""
    print("case: draft", io, dk, dv, B, T, H, Hk, flush=True)
    raw = T % 2 == 0
    x = _draft_inputs(B + T, (B, T), B, H, Hk, dk, dv, io, raw)
    flags = gdn.GDN_QK_L2NORM | gdn.GDN_GATE_LOGITS if raw else 0
    some = np.random.default_rng(T).integers(0, T + 1, B)
    for keep in (None, [0] * B, some, [T + 5] * B, [-1] * B):
        S = x[5].clone()
        o = gdn.gdn_draft_step(*x[:5], S, keep=None if keep is None else i32(keep), flags=flags, scale=0.5)
        _check_draft(x, o, S, keep, None, T, io, raw, "keep %s" % (keep if keep is None else list(keep)[:4]), 0.5)
        S2 = x[5].clone()
        assert gdn.gdn_draft_step(None, *x[1:5], S2, keep=None if keep is None else i32(keep), flags=flags) is None
        _check_draft(x, None, S2, keep, None, T, io, raw, "  state alone")
        if keep is not None and max(keep) <= 0:
            assert torch.equal(S, x[5]) and torch.equal(S2, x[5])


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_draft_step_packed(io):
    """Sequences of no token, of several tiles; rows behind the last sequence stay; offsets outside the contract are clamped."""
    cu = [0, 3, 3, 20, 12, 29, 30]
    T, n, H = 34, 6, 4
    x = _draft_inputs(7, (1, T), n, H, 2, 128, 128, io, False)
    keep = [2, 4, 17, 0, 8, 1]
    S, o = x[5].clone(), torch.full_like(x[2], 7.0)
    gdn.gdn_draft_step(*x[:5], S, keep=i32(keep), cu_seqlens=i32(cu), o=o)
    assert (o[0, 30:] == 7).all()
    _check_draft(x, o, S, keep, cu, T, io, False, "packed")
    cu = [0] + list(np.cumsum(np.random.default_rng(3).integers(0, 4, 150)))
    x = _draft_inputs(8, (1, max(cu) + 3), 150, 4, 4, 64, 64, io, True)
    S = x[5].clone()
    o = gdn.gdn_draft_step(*x[:5], S, cu_seqlens=i32(cu), flags=gdn.GDN_QK_L2NORM | gdn.GDN_GATE_LOGITS)
    _check_draft(x, o, S, None, cu, 3, io, True, "150 sequences")


def test_draft_step_keeps_what_is_not_kept_out():
    """Drafts that are not kept bring values that are not finite, and gates of 0: earlier outputs and the state stay clean;
    a state row that is not finite stays by itself."""
    x = _draft_inputs(9, (2, 10), 2, 2, 2, 128, 128, "f32", False)
    x[3][0, 1] = -float("inf")                            # everything before is forgotten
    clean = [y.clone() for y in x]
    for y in (x[0], x[1], x[2], x[3], x[4]):
        y[0, 4:] = float("nan")
        y[1, 9:] = float("inf")
    S = x[5].clone()
    o = gdn.gdn_draft_step(*x[:5], S, keep=i32([4, 9]))
    assert torch.isfinite(S).all() and torch.isfinite(o[0, :4]).all() and torch.isfinite(o[1, :9]).all()
    want_o, want_S = drafts.draft_step(*[f64(y) for y in clean], keep=[4, 9])
    assert np.abs(f64(S) - want_S).max() < 2e-4 and np.abs(f64(o)[0, :4] - want_o[0, :4]).max() < 2e-4
    S = clean[5].clone()
    S[1, 0, 5, 3] = float("inf")
    o = gdn.gdn_draft_step(*clean[:5], S)
    bad = ~torch.isfinite(S)
    assert bad[1, 0, 5].any() and not bad[0].any() and not bad[1, 1].any() and not bad[1, 0, :5].any() and not bad[1, 0, 6:].any()
    bad = ~torch.isfinite(o)
    assert bad[1, :, 0, 5].any() and bad.sum() == bad[1, :, 0, 5].sum()


def test_draft_step_matches_decode_steps():
    """Token by token through gdn_decode_step_ex: both within fp32 roundings of the other."""
    x = _draft_inputs(11, (3, 6), 3, 4, 2, 128, 128, "f32", True)
    flags = gdn.GDN_QK_L2NORM | gdn.GDN_GATE_LOGITS
    S, S1 = x[5].clone(), x[5].clone()
    o = gdn.gdn_draft_step(*x[:5], S, flags=flags)
    for t in range(6):
        y = gdn.gdn_decode_step_ex(*[z[:, t].contiguous() for z in x[:5]], S1, flags=flags)
        assert (y - o[:, t]).abs().max() < 1e-4
    assert (S - S1).abs().max() < 1e-4


# ------------------------------------------------------------------ gdn_draft_verify
def _verify_inputs(seed, n, m, V, io):
    r = np.random.default_rng(seed)
    logits = 2 * r.standard_normal((n, m + 1, V))
    soft = lambda y: np.exp(y) / np.exp(y).sum(-1, keepdims=True)   # noqa: E731
    p = torch.from_numpy(soft(logits)).to(IO[io])
    q = torch.from_numpy(soft(logits[:, :m] + 0.5 * r.standard_normal((n, m, V)))).to(IO[io])
    x = np.array([[r.choice(V, p=soft(logits[i, j])) for j in range(m)] for i in range(n)]).reshape(n, m)
    return p, q, torch.from_numpy(x).int(), torch.from_numpy(r.random((n, m + 1))).float()


def _verify(p, q, x, lens, u, **kw):
    m = u.shape[1] - 1
    t, c = gdn.gdn_draft_verify(p.cuda(), u.cuda(), drafts=x.cuda() if m else None, q=None if q is None or not m else q.cuda(),
                                draft_lens=None if lens is None else i32(lens), **kw)
    wt, wc = drafts.verify(f64(p.float()), None if q is None else f64(q.float()), ints(x), lens, f64(u))
    assert (ints(t) == wt).all() and (ints(c) == wc).all(), (ints(t), wt)
    return t, c


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("n,m,V", [(1, 1, 1), (1, 0, 5), (3, 2, 7), (5, 4, 257), (2, 3, 4096), (2, 2, 4097), (3, 5, 9001), (70, 1, 50)])
def test_verify(io, n, m, V):
    print("case: verify", io, n, m, V, flush=True)
    p, q, x, u = _verify_inputs(n + V, n, m, V, io)
    _verify(p, q, x, None, u)
    _verify(p, None, x, None, u)
    if m:
        _verify(p, q, x, np.random.default_rng(1).integers(-1, m + 2, n), u)
        u[:, 0] = 1.0                                     # the first draft mostly not taken
        _verify(p, q, x, None, u)


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_verify_borders(io):
    """Random numbers on the border of acceptance and of a sum, 0, the largest below 1, and outside [0, 1)."""
    p = torch.tensor([[[.5, .25, .25, 0.]] * 2] * 12).to(IO[io])
    q = torch.tensor([[[.25, .5, .25, 0.]]] * 12).to(IO[io])
    x = torch.tensor([[1]] * 12, dtype=torch.int32)
    u = torch.tensor([[.5, 0], [np.nextafter(np.float32(.5), np.float32(0)), 0], [.5, .999], [0, .5], [0, .75], [0, .25], [0, 1], [0, 5], [0, -1],
                      [0, float("nan")], [float("nan"), .5], [0, np.nextafter(np.float32(1), np.float32(0))]]).float()
    t, c = _verify(p, q, x, None, u)
    assert ints(t)[:6].tolist() == [[0, -1], [1, 0], [0, -1], [1, 1], [1, 2], [1, 0]] and ints(t)[6:8, 1].tolist() == [2, 2]


def test_verify_odd_values():
    """Zero rows, equal rows, entries that are negative, infinite or NaN, drafts outside the vocabulary, a draft that its own
    model gives nothing."""
    p, q, x, u = _verify_inputs(5, 9, 2, 300, "f32")
    p[0] = 0
    q[1] = p[1, :2]                                       # (every draft taken but for u q = p, then from p itself)
    u[1, 0] = 1.0
    p[2, :, 5], q[3, :, 7], p[4, :, 9] = float("nan"), float("nan"), float("inf")
    p[5, :, ::2] = -1.0
    x[6] = torch.tensor([300, -1], dtype=torch.int32)
    q[7, 0, x[7, 0]] = 0
    p[8, :, :] = 0
    p[8, :, 299] = 1e-30
    u[8, 0] = 0.9
    _verify(p, q, x, None, u)
    _verify(p, None, x, None, u)


def test_verify_rows_of_a_padded_vocabulary():
    """Parts of wider rows, odd strides and odd starts, given outputs and workspace."""
    for io in ("f32", "bf16"):
        p, q, x, u = _verify_inputs(6, 4, 3, 5001, io)
        wide = [torch.full((4, y.shape[1], 5011), 9.0, dtype=IO[io]).cuda() for y in (p, q)]
        for y, w in zip((p, q), wide):
            w[..., 3:5004] = y.cuda()
        t, c = torch.full((4, 4), 9, dtype=torch.int32).cuda(), torch.full((4,), 9, dtype=torch.int32).cuda()
        ws = torch.empty(gdn.gdn_draft_verify_workspace_bytes(4, 3, 5001), dtype=torch.uint8, device="cuda")
        got = gdn.gdn_draft_verify(wide[0][..., 3:5004], u.cuda(), drafts=x.cuda(), q=wide[1][..., 3:5004], tokens=t, counts=c, workspace=ws)
        assert got[0] is t and got[1] is c
        wt, wc = drafts.verify(f64(p.float()), f64(q.float()), ints(x), None, f64(u))
        assert (ints(t) == wt).all() and (ints(c) == wc).all()


def test_verify_large_vocabulary():
    """131072 and 100003 tokens, 80-bit sums on the host."""
    for n, m, V, io in ((3, 2, 131072, "f32"), (2, 1, 100003, "bf16")):
        p, q, x, u = _verify_inputs(7, n, m, V, io)
        u[0, 0] = 1.0
        t, c = gdn.gdn_draft_verify(p.cuda(), u.cuda(), drafts=x.cuda(), q=q.cuda())
        P, Q = f64(p.float()), f64(q.float())
        for s in range(n):
            j = 0
            while j < m and float(u[s, j]) * Q[s, j, x[s, j]] < P[s, j, x[s, j]]:
                j += 1
            w = np.maximum(P[s, j] - Q[s, j], 0) if j < m else P[s, j]
            sums = np.cumsum(w.astype(np.longdouble))
            want = int(np.searchsorted(sums, np.longdouble(float(u[s, m])) * sums[-1], side="right"))
            assert ints(c)[s] == j + 1 and ints(t)[s].tolist() == ints(x)[s, :j].tolist() + [want] + [-1] * (m - j)
