"""How gdn_attention_paged cuts a step into items, written out on the host after its comments in gdn.hip and paged.hip, in the
same float32 steps: for tests of the rule's bounds, and so that a test can say which of its branches a case takes."""
import numpy as np

UNIT, CUS = 128, 256
F = np.float32


def plan(B, T, H, Hkv, page, max_pages, n_seqs):
    """The host's part: rows per block, row blocks and items per key/value head at most, and round, fine, spare."""
    G = H // Hkv
    few = T * G // 16 + min(n_seqs, T) if n_seqs else B * -(-T * G // 16)
    rb = 16 if T * G <= 16 * max(n_seqs, 1) or few * Hkv <= 32 else 128
    blocks = T * G // rb + min(n_seqs, T) if n_seqs else B * -(-T * G // rb)
    units = -(-page * max_pages // UNIT)
    round_ = max(1, 2 * CUS // Hkv)
    if rb == 16:
        fine, most = 8, 8 * CUS // Hkv
        spare = max(0, min(most - blocks, blocks * units // fine))
        items = max(blocks + spare, min(round_, blocks * units))
        if units == 1:
            spare = 0
    else:
        fine = 1 << 23
        items = max(blocks, min(round_, blocks * units))
        spare = items - blocks if items > blocks + blocks // 4 else 0
    return dict(rb=rb, blocks=blocks, items=items if spare else blocks, round=round_, fine=fine, spare=spare, G=G, cap=page * max_pages)


def workspace(p, Hkv, d):
    if p["spare"] == 0:
        return 0
    rows = p["items"] * Hkv * p["rb"]
    return -(-rows * 8 // 256) * 256 + rows * d * 4


def cut(p, new, lens):
    """The device's part: units per chunk, how that came about (times it grew; whether it fell back), and every sequence's
    (row blocks, units)."""
    seqs = [(-(-n * p["G"] // p["rb"]), max(-(-min(max(L, 0), p["cap"]) // UNIT), 1)) for n, L in zip(new, lens)]
    if p["spare"] == 0:
        return 1 << 23, 0, False, seqs
    lanes = np.zeros(64, dtype=F)
    for base in range(0, len(seqs), 64):
        for i, (b, u) in enumerate(seqs[base:base + 64]):
            lanes[i] = lanes[i] + F(b) * F(u)
    for off in (1, 2, 4, 8, 16, 32):
        lanes = lanes + lanes[np.arange(64) ^ off]
    total = F(lanes[0] * F(1 - 2.0 ** -19))
    up = lambda x: int(min(np.ceil(F(x)), F(2 ** 23)))   # noqa: E731
    count = lambda c: sum(b * -(-u // c) for b, u in seqs)   # noqa: E731
    uneven = lambda c: c > p["fine"] and total < F(F(0.8) * F(c)) * F(p["round"])   # noqa: E731
    c, grown = max(up(total / F(p["round"])), 1 if p["rb"] == 16 else 4), 0
    while True:
        fits = count(c) <= p["round"]
        if fits or c >= 1 << 23 or uneven(c):
            break
        c, grown = c + (c + 7) // 8, grown + 1
    fell = not fits or uneven(c)
    if fell:
        c = max(up(F(total * F(1 + 2.0 ** -17)) / F(p["spare"])), p["fine"])
    return min(c, 1 << 23), grown, bool(fell), seqs


def items(p, new, lens):
    """Every (sequence, row block, chunk) that has work, as its item's number, and the number of items that the rule makes."""
    c, _, _, seqs = cut(p, new, lens)
    first, out = 0, []
    for s, (blocks, units) in enumerate(seqs):
        L = max(lens[s], 0)
        for rb in range(blocks):
            i = min((rb * p["rb"] + p["rb"] - 1) // p["G"], new[s] - 1)
            end = min(max(L - new[s] + i + 1, 0), p["cap"])
            chunks = 1
            if end > c * UNIT:
                chunks = -(-end // (c * UNIT))
                size = -(-(-(-end // chunks)) // UNIT) * UNIT
                chunks = -(-end // size)
            for j in range(chunks):
                out.append(first + j * blocks + (rb if j % 2 else blocks - 1 - rb))
        first += blocks * -(-units // c)
    return out, first
