"""A serving step of drafted tokens over shared prompts: what is measured, plain forms, and exact values to hold both against.

Four operators, in the order in which a step calls them:

  tables   the pages that a step's sequences need, taken from and given back to a pool on the GPU, with the step's packed
           offsets, positions and cache slots
  shared   the new tokens' attention over the paged cache where groups of sequences share a long prefix
  draft    the recurrent layers over a few drafted tokens a sequence: all outputs, and the state after the kept ones
  verify   which drafted tokens the target's probabilities accept, and the token that follows them, from given random numbers

``listed()`` names twelve cases, ``draw(rng)`` gives others of the same ranges: 1 to 512 sequences, drafts of 0 to 15 tokens,
prefixes of up to 65536 tokens and up to 4096 of a sequence's own behind them, vocabularies of 1000 to 200000.
"""
from __future__ import annotations

import math
import random

import torch

own = False

E4M3 = torch.float8_e4m3fn
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": E4M3}
L2_EPS = 1e-6


def _tables(name, n, new, old, *, page=64, shared=0, leave=False, dense=False, mix=0):
    """``new``, ``old``: the ranges that the sequences' tokens are spread over; ``shared``: pages at the front of every
    sequence that are no page of its own; ``leave``: every second sequence ends at the end of the step."""
    return dict(name=name, op="tables", n=n, new_lo=new[0], new_hi=new[1], old_lo=old[0], old_hi=old[1], page=page,
                shared=shared, leave=leave, dense=dense, mix=mix)


def _shared(name, n, prefix, tail, new=(1, 1), *, groups=1, H=16, Hkv=8, d=128, page=64, cache="bf16", empty=0, mix=0):
    """``prefix``: tokens that the sequences of a group share; ``tail``: a sequence's own before the step; ``empty``: sequences
    without any token, which fill a batch up."""
    return dict(name=name, op="shared", n=n, groups=groups, prefix_lo=prefix[0], prefix_hi=prefix[1], tail_lo=tail[0],
                tail_hi=tail[1], new_lo=new[0], new_hi=new[1], H=H, Hkv=Hkv, d=d, page=page, cache=cache, empty=empty, mix=mix)


def _draft(name, n, new, *, H=16, Hk=16, dk=128, dv=128, io="bf16", keep="some", outputs=True, raw=False, mix=0):
    """``keep``: tokens whose update stays in the state: none, some of them, or all; ``raw``: q and k of any length, gates as
    logits."""
    return dict(name=name, op="draft", n=n, new_lo=new[0], new_hi=new[1], H=H, Hk=Hk, dk=dk, dv=dv, io=io, keep=keep,
                outputs=outputs, raw=raw, mix=mix)


def _verify(name, n, m, V, *, io="f32", q=True, ragged=False, sharp=2.0, mix=0):
    """``q``: whether the drafts come with probabilities (else each is certain); ``sharp``: the logits' spread."""
    return dict(name=name, op="verify", n=n, m=m, V=V, io=io, q=q, ragged=ragged, sharp=sharp, mix=mix)


def listed():
    return [
        # a serving batch's next step of five tokens, small pages: some sequences start a page, some give it back
        _tables("tables_b256", 256, (5, 5), (16, 8191), page=16, mix=1),
        # a batch of prompts behind a shared system prompt, every second one ends after the step: maps of many tokens
        _tables("tables_prompts", 8, (512, 4096), (0, 4000), page=32, shared=40, leave=True, mix=2),
        # a few users of one system prompt, next token: latency
        _shared("shared_b8_bf16", 8, (1000, 1000), (1, 300), mix=3),
        # a serving batch behind a long instruction, next token
        _shared("shared_b64_bf16", 64, (8192, 8192), (64, 2000), mix=4),
        # questions on one very long document, 8-bit cache
        _shared("shared_document_e4m3", 48, (65536, 65536), (16, 500), cache="e4m3", mix=5),
        # drafted tokens to verify, four tenants with a prompt each, uneven drafts, a batch not quite full
        _shared("shared_groups_draft", 36, (2000, 16384), (30, 4000), (2, 6), groups=4, Hkv=4, page=16, empty=2, mix=6),
        # one user's drafted tokens: outputs only, the state stays until they are verified
        _draft("draft_b1_f32", 1, (5, 5), io="f32", keep="none"),
        # a serving batch's drafted tokens, the accepted ones' update kept in the same pass
        _draft("draft_b64_bf16", 64, (5, 5), mix=7),
        # the kept tokens alone, after their verification, uneven drafts, grouped key heads, transforms in the kernel
        _draft("draft_keep_b128_bf16", 128, (1, 9), H=16, Hk=4, outputs=False, raw=True, mix=8),
        # one user's four drafts
        _verify("verify_b1_f32", 1, 4, 50000, mix=9),
        # a serving batch's drafts, large vocabulary
        _verify("verify_b64_f32", 64, 4, 131072, mix=10),
        # uneven drafts found without a model (each certain), an odd vocabulary in bf16
        _verify("verify_b96_bf16", 96, 7, 100003, io="bf16", q=False, ragged=True, mix=11),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(max(1, lo)), math.log(max(1, hi))))))


def draw(rng):
    op, mix = rng.choice(["tables", "shared", "shared", "draft", "verify"]), rng.randrange(100000)
    if op == "tables":
        page, shared = rng.choice([16, 32, 64, 128]), rng.choice([0, 0, rng.randint(1, 64)])
        if rng.random() < 0.6:
            new = rng.randint(1, 16)
            return _no_name(_tables("", _log_int(rng, 1, 512), (new, new), (0, _log_int(rng, 16, 8192)), page=page, shared=shared,
                                    leave=rng.random() < 0.3, dense=rng.random() < 0.5, mix=mix))
        n = rng.randint(1, 8)
        top = _log_int(rng, 8, 4096)
        return _no_name(_tables("", n, (max(1, top // rng.choice([1, 4, 40])), top), (0, _log_int(rng, 16, 4096)), page=page,
                                shared=shared, leave=rng.random() < 0.5, mix=mix))
    if op == "shared":
        H, d = rng.choice([8, 16, 16, 32]), rng.choice([64, 128, 128])
        Hkv, page = rng.choice([h for h in (2, 4, 8, 16) if h <= H]), rng.choice([16, 32, 64, 128])
        n, room = _log_int(rng, 2, 128), 48 * 16 * 128 / (H * d)       # (sequences with the largest listed prefix)
        groups = rng.choice([1, 1, min(n, rng.randint(2, 6))])
        new = rng.choice([(1, 1), (1, 1), (4, 4), (1, 8)])
        rows = n * (new[0] + new[1]) / 2
        most = int(65536 * min(1.0, room / rows, 8 * 128 / (Hkv * d) / groups * (1 if rows >= 16 else 0.5)))
        top = _log_int(rng, 16, max(64, most))
        tail = _log_int(rng, 1, max(4, min(4096, 60000 * 1024 // (Hkv * d) // n)))
        return _no_name(_shared("", n, (max(0, top // rng.choice([1, 4])), top), (tail // rng.choice([1, 4, 16]), tail), new,
                                groups=groups, H=H, Hkv=Hkv, d=d, page=page, cache=rng.choice(["bf16", "e4m3"]),
                                empty=rng.choice([0, 0, rng.randint(1, 4)]), mix=mix))
    if op == "draft":
        H, dk, dv = rng.choice([2, 8, 16, 32]), rng.choice([64, 128, 128]), rng.choice([64, 128, 128])
        hi = rng.randint(1, 16)
        return _no_name(_draft("", _log_int(rng, 1, 128 * 16 // H), (rng.choice([hi, max(1, hi // 3)]), hi), H=H,
                               Hk=rng.choice([h for h in (1, 2, 4, 16) if h <= H]), dk=dk, dv=dv, io=rng.choice(["f32", "bf16"]),
                               keep=rng.choice(["none", "some", "all"]), outputs=rng.random() < 0.7, raw=rng.random() < 0.5, mix=mix))
    m, V = rng.randint(0, 8), _log_int(rng, 1000, 200000)
    n = _log_int(rng, 1, max(1, min(256, 64 * 5 * 131072 // ((m + 1) * V))))
    return _no_name(_verify("", n, m, V, io=rng.choice(["f32", "bf16"]), q=rng.random() < 0.7, ragged=rng.random() < 0.5,
                            sharp=rng.choice([0.5, 2.0, 6.0]), mix=mix))


def _no_name(case):
    del case["name"]
    return case


# ------------------------------------------------------------------ inputs

def _spread(case, n, what, rng):
    """n numbers spread over the logarithm of the range ``what`` of the case."""
    lo, hi = case[what + "_lo"], case[what + "_hi"]
    return [_log_int(rng, lo + 1, hi + 1) - 1 for _ in range(n)]


def _sizes(case):
    """The case's own whole numbers, the same for every seed."""
    rng = random.Random(case["mix"])
    n = case["n"]
    if case["op"] == "tables":
        new, old = _spread(case, n, "new", rng), _spread(case, n, "old", rng)
        old = [a + case["shared"] * case["page"] for a in old]
        after = [0 if case["leave"] and i % 2 else old[i] + rng.randint(1, new[i]) for i in range(n)]
        return new, old, after
    if case["op"] == "shared":
        g = case["groups"]
        cuts = sorted(rng.sample(range(1, n), g - 1)) if g > 1 else []
        prefix, tail, new = _spread(case, g, "prefix", rng), _spread(case, n, "tail", rng), _spread(case, n, "new", rng)
        empty = set(rng.sample(range(n), min(case["empty"], n - 1)))
        return [0] + cuts + [n], prefix, tail, new, empty
    if case["op"] == "draft":
        new = _spread(case, n, "new", rng)
        keep = [0 if case["keep"] == "none" else a if case["keep"] == "all" else rng.randint(0, a) for a in new]
        return new, keep
    return [rng.randint(0, case["m"]) if case["ragged"] else case["m"] for _ in range(n)]


class _Make:
    """Values on the GPU from a seed."""

    def __init__(self, seed):
        self.dev = torch.device("cuda", torch.cuda.current_device())
        self.rng = torch.Generator(device=self.dev)
        self.rng.manual_seed(seed)

    def normal(self, *shape):
        return torch.randn(shape, generator=self.rng, device=self.dev, dtype=torch.float32)

    def uniform(self, *shape):
        return torch.rand(shape, generator=self.rng, device=self.dev, dtype=torch.float32)

    def order(self, n):
        return torch.randperm(n, generator=self.rng, device=self.dev).to(torch.int32)

    def ints(self, values):
        return torch.tensor(values, dtype=torch.int32).to(self.dev)


def _offsets(counts):
    return [sum(counts[:i]) for i in range(len(counts) + 1)]


def _tables_inputs(case, seed):
    """A pool and tables as the step before left them."""
    mk, (new, old, after), page, n, shared = _Make(seed), _sizes(case), case["page"], case["n"], case["shared"]
    first = torch.tensor([max(-(-a // page), shared) for a in after])          # pages held before the step
    most = max(-(-(a + b) // page) for a, b in zip(old, new)) + 2
    need = sum(max(0, -(-(a + b) // page) - shared) for a, b in zip(old, new))
    n_pages = shared + need + 7
    order = mk.order(n_pages)
    entry = torch.arange(most)
    mine = (entry >= shared) & (entry < first[:, None])
    at = shared + torch.cumsum(mine.flatten(), 0).view(mine.shape) - 1
    at = torch.where(mine, at, torch.where(entry < shared, entry, -1))
    table = torch.where((at >= 0).to(mk.dev), order[at.clamp(min=0).to(mk.dev)], order.new_full((), -1))
    used = shared + int(mine.sum())
    free = torch.full_like(order, -1)
    free[:n_pages - used] = order[used:]
    rows = sum(new) if not case["dense"] else n * new[0]
    shape = (n, new[0]) if case["dense"] else (rows,)
    return dict(
        case=case, lens=mk.ints([a + b for a, b in zip(old, new)]), after=mk.ints(after),
        new_lens=None if case["dense"] else mk.ints(new), shared=mk.ints([shared] * n) if shared else None,
        table=table.contiguous(), held=first.to(torch.int32).to(mk.dev), free=free, n_free=mk.ints([n_pages - used]),
        missing=mk.ints([0]), cu=mk.ints([0] * (n + 1)), positions=torch.zeros(shape, dtype=torch.int32, device=mk.dev),
        slots=torch.zeros(shape, dtype=torch.int64, device=mk.dev))


def _shared_inputs(case, seed):
    """Queries, the cache with its tables: the first prefix // page pages of a group's sequences are the same ones."""
    mk, (cuts, prefix, tail, new, empty) = _Make(seed), _sizes(case)
    n, H, Hkv, d, page = (case[x] for x in ("n", "H", "Hkv", "d", "page"))
    group = [sum(i >= c for c in cuts[1:]) for i in range(n)]
    common = [p // page for p in prefix]
    lens = [0 if i in empty else prefix[group[i]] + tail[i] + new[i] for i in range(n)]
    own_pages = [0 if i in empty else -(-lens[i] // page) - common[group[i]] for i in range(n)]
    n_pages = sum(common) + sum(own_pages) + 3
    width = max(max(common) + 1, max(common[g] + o for g, o in zip(group, own_pages)) + 1)
    order, entry, at = mk.order(n_pages), torch.arange(width), torch.full((n, width), -1)
    c, base = torch.tensor([common[g] for g in group])[:, None], torch.tensor(_offsets(common))[torch.tensor(group)][:, None]
    mine = torch.tensor(_offsets(own_pages)[:-1])[:, None] + sum(common)
    at = torch.where(entry < c, base + entry, torch.where(entry < c + torch.tensor(own_pages)[:, None], mine + entry - c, at))
    at[sorted(empty)] = -1
    for g in range(len(prefix)):      # (a group's first sequence names the shared pages, also where it is empty)
        at[cuts[g], :common[g]] = torch.arange(_offsets(common)[g], _offsets(common)[g + 1])
    x = dict(case=case, block_table=torch.where((at >= 0).to(mk.dev), order[at.clamp(min=0).to(mk.dev)], order.new_full((), -1)),
             seq_lens=mk.ints(lens), prefix_lens=mk.ints(prefix), cu_groups=mk.ints(cuts) if case["groups"] > 1 else None)
    dense = case["new_lo"] == case["new_hi"]
    x["cu"] = None if dense else mk.ints(_offsets(new))
    x["q"] = mk.normal(*((n, new[0]) if dense else (1, sum(new))), H, d).bfloat16()
    for name in ("k", "v"):
        values = mk.normal(n_pages, Hkv, page, d)
        if case["cache"] == "bf16":
            x[name + "_cache"], x[name + "_scale"] = values.bfloat16(), None
        else:   # values of about unit size, each page and head with a power of two of its own
            scale = torch.exp2(torch.floor(mk.normal(n_pages, Hkv)) - 6)
            x[name + "_cache"] = (values / scale[..., None, None]).clamp(-448, 448).to(E4M3)
            x[name + "_scale"] = scale
    x["o"] = torch.empty_like(x["q"])
    return x


def _draft_inputs(case, seed):
    """A few tokens a sequence (the last one chosen and the drafts behind it) and the states before them."""
    mk, (new, keep) = _Make(seed), _sizes(case)
    n, H, Hk, dk, dv, io = (case[x] for x in ("n", "H", "Hk", "dk", "dv", "io"))
    dense = case["new_lo"] == case["new_hi"]
    rows = (n, new[0]) if dense else (1, sum(new))
    q, k, v = mk.normal(*rows, Hk, dk), mk.normal(*rows, Hk, dk), mk.normal(*rows, H, dv)
    beta, g = mk.normal(*rows, H), mk.normal(*rows, H) + 2
    if not case["raw"]:
        q, k = (y / torch.linalg.vector_norm(y, dim=-1, keepdim=True) for y in (q, k))
        beta, g = 1 / (1 + torch.exp(-beta)), -torch.log1p(torch.exp(g))
    x = dict(case=case, q=q.to(DTYPES[io]), k=k.to(DTYPES[io]), v=v.to(DTYPES[io]), g=g, beta=beta, S=0.1 * mk.normal(n, H, dv, dk),
             keep=mk.ints(keep), cu=None if dense else mk.ints(_offsets(new)))
    x["o"] = torch.empty_like(x["v"]) if case["outputs"] else None
    return x


def _verify_inputs(case, seed):
    """Probabilities of the target and, a little off them, of the model that drafted; drafts drawn from the latter."""
    mk, lens = _Make(seed), _sizes(case)
    n, m, V = case["n"], case["m"], case["V"]
    logits = case["sharp"] * mk.normal(n, m + 1, V)
    x = dict(case=case, p=torch.softmax(logits, -1).to(DTYPES[case["io"]]), q=None, u=mk.uniform(n, m + 1), drafts=None,
             lens=mk.ints(lens) if case["ragged"] else None)
    if m:
        q = torch.softmax(logits[:, :m] + 0.5 * mk.normal(n, m, V), -1)
        drawn = (torch.cumsum(q, -1) < mk.uniform(n, m, 1)).sum(-1).clamp(max=V - 1)
        x["drafts"] = (drawn if case["q"] else torch.where(mk.uniform(n, m) < 0.7, q.argmax(-1), drawn)).to(torch.int32)
        x["q"] = q.to(DTYPES[case["io"]]) if case["q"] else None
    x["tokens"] = torch.zeros(n, m + 1, dtype=torch.int32, device=mk.dev)
    x["counts"] = torch.zeros(n, dtype=torch.int32, device=mk.dev)
    return x


def prepare(case, seed):
    """A step's inputs, and the buffers that a serving program keeps from step to step."""
    return {"tables": _tables_inputs, "shared": _shared_inputs, "draft": _draft_inputs, "verify": _verify_inputs}[case["op"]](case, seed)


# ------------------------------------------------------------------ the plain forms

def _plain_call(x, lens, maps):
    """One call of the tables' operator: pages given back, then taken, in order of sequence and entry; then the maps."""
    table, free, page = x["table"], x["free"], x["case"]["page"]
    n, width = table.shape
    n_pages, n_free = free.numel(), x["n_free"].long()
    length, held = lens.long().clamp(min=0)[:, None], x["held"].long().clamp(0, width)[:, None]
    fixed = torch.zeros_like(held) if x["shared"] is None else torch.minimum(x["shared"].long()[:, None], held)
    target = torch.maximum(((length + page - 1) // page).clamp(max=width), fixed)
    entry = torch.arange(width, device=table.device)
    give, take = (entry >= target) & (entry < held), (entry >= held) & (entry < target)
    rank = torch.cumsum(give.flatten(), 0).view(give.shape) - 1
    pool = torch.cat([free, free.new_zeros(1)])                    # (its last entry takes what is not given)
    pool.scatter_(0, torch.where(give, n_free + rank, n_pages).flatten(), table.flatten())
    full = n_free + give.sum()
    got = torch.minimum(take.sum(), full)
    rank = torch.cumsum(take.flatten(), 0).view(take.shape) - 1
    found = take & (rank < got)
    page_of = pool[torch.where(found, full - got + rank, 0)]
    table.copy_(torch.where(found, page_of, torch.where(give | take, -1, table)))
    x["held"].copy_((torch.minimum(held, target)[:, 0] + found.sum(1)).int())
    free.copy_(pool[:-1])
    x["n_free"].copy_((full - got).int())
    x["missing"].copy_((take.sum() - got).int())
    if not maps:
        return
    rows = x["slots"].numel()
    t = torch.arange(rows, device=table.device)
    if x["new_lens"] is None:
        cu = torch.arange(n + 1, device=table.device) * (rows // n)
    else:
        cu = torch.cat([t.new_zeros(1), torch.cumsum(x["new_lens"].long().clamp(min=0), 0)]).clamp(max=rows)
    s = torch.searchsorted(cu[1:], t, right=True)
    inside, s = s < n, s.clamp(max=n - 1)
    pos = length[s, 0] - cu[s + 1] + t
    block = pos // page
    there = inside & (pos >= 0) & (block < width)
    page_id = torch.where(there, table[s, block.clamp(0, width - 1)], -1).long()
    x["cu"].copy_(cu.int())
    x["positions"].copy_(torch.where(inside, pos, 0).int().view(x["positions"].shape))
    x["slots"].copy_(torch.where(page_id >= 0, page_id * page + pos % page, -1).view(x["slots"].shape))


def _plain_tables(x):
    _plain_call(x, x["lens"], True)
    _plain_call(x, x["after"], False)


def _tables_out(x):
    return {c: x[c] for c in ("cu", "positions", "slots", "table", "held", "free", "n_free", "missing")}


def _counts(x, n):
    """New tokens of every sequence, and of every token of the call its sequence and place."""
    rows = x["q"].shape[0] * x["q"].shape[1]
    t = torch.arange(rows, device=x["q"].device)
    if x["cu"] is None:
        T = rows // n
        return torch.full((n,), T, device=t.device), t // T, t % T
    cu = x["cu"].long()
    s = (t[:, None] >= cu[1:]).sum(1)
    return cu[1:] - cu[:-1], s, t - cu[s]


def _gathered(x, name, ids):
    """Keys or values of pages ids [n, pages] in float32, [n, H_kv, pages * page, d]."""
    y, ids = x[name + "_cache"], ids.long().clamp(min=0)
    y = (y.view(torch.uint8)[ids].view(E4M3) if y.dtype == E4M3 else y[ids]).float()
    if x[name + "_scale"] is not None:
        y = y * x[name + "_scale"][ids][..., None, None]
    return y.transpose(1, 2).flatten(2, 3)


def _plain_shared(x):
    """Scores of a group's rows with its prefix in one product, of every sequence's rows with its own keys in another."""
    case, (cuts, prefix, tail, new, empty) = x["case"], _sizes(x["case"])
    n, H, Hkv, d, page, ng = (case[c] for c in ("n", "H", "Hkv", "d", "page", "groups"))
    G, most, dev = H // Hkv, max(new), x["q"].device
    count, s, i = _counts(x, n)
    group = torch.tensor([sum(j >= c for c in cuts[1:]) for j in range(n)]).to(dev)
    place = torch.arange(n, device=dev) - torch.tensor(cuts).to(dev)[group]
    wide = max(b - a for a, b in zip(cuts, cuts[1:]))
    q = torch.zeros(n, most, H, d, device=dev)
    q[s, i] = x["q"].flatten(0, 1).float()
    q = q.view(n, most, Hkv, G, d).permute(0, 2, 1, 3, 4).flatten(2, 3) / math.sqrt(d)          # [n, H_kv, rows, d]
    whole = x["prefix_lens"].long() // page                                                    # pages of each group's prefix
    first = x["block_table"][torch.tensor(cuts[:-1]).to(dev)]
    together = torch.zeros(ng, wide, *q.shape[1:], device=dev)
    together[group, place] = q
    together = together.transpose(1, 2).flatten(2, 3)                                          # [groups, H_kv, rows, d]
    pages = max(max(p // page for p in prefix), 1)
    k, v = _gathered(x, "k", first[:, :pages]), _gathered(x, "v", first[:, :pages])
    hide = torch.arange(k.shape[2], device=dev) >= whole[:, None] * page
    score = torch.matmul(together, k.transpose(2, 3).contiguous()).masked_fill_(hide[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True).clamp(min=-1e30)
    e = torch.exp_(score.sub_(top))
    of = lambda y: y.view(ng, Hkv, wide, -1, y.shape[-1])[group, :, place]                     # noqa: E731  back to [n, H_kv, rows, ..]
    m1, l1, o1 = of(top), of(e.sum(-1, keepdim=True)), of(torch.matmul(e, v))
    # every sequence's own keys
    width = x["block_table"].shape[1]
    span = max(1, max(-(-(0 if j in empty else (prefix[g] % page + tail[j] + new[j])) // page) for j, g in enumerate(group.tolist())))
    col = whole[group][:, None] + torch.arange(span, device=dev)
    ids = torch.where(col < width, x["block_table"].gather(1, col.clamp(max=width - 1)).long(), -1)
    k, v = _gathered(x, "k", ids), _gathered(x, "v", ids)
    score = torch.matmul(q, k.transpose(2, 3).contiguous())
    last = (x["seq_lens"].long() - count)[:, None] + torch.arange(most, device=dev)            # a row's own position
    key = (whole * page)[group][:, None] + torch.arange(k.shape[2], device=dev)
    seen = (key[:, None] <= last[..., None]).repeat_interleave(G, 1)[:, None]
    score = torch.where(seen, score, -math.inf)
    m2 = score.amax(-1, keepdim=True).clamp(min=-1e30)
    e = torch.exp(score - m2)
    none = (x["seq_lens"] == 0)[:, None, None, None]
    m = torch.maximum(torch.where(none, m2, m1), m2)
    a, b = torch.where(none, 0.0, torch.exp(m1 - m)), torch.exp(m2 - m)
    total = a * l1 + b * e.sum(-1, keepdim=True)
    o = (a * o1 + b * torch.matmul(e, v)) / torch.where(total == 0, 1.0, total)
    o = o.view(n, Hkv, most, G, d).permute(0, 2, 1, 3, 4).flatten(2, 3)
    return o[s, i].bfloat16().view(x["q"].shape)


def _plain_draft(x):
    """The tokens' products with the state before them in one product each; what they add to one another by a unit triangular
    system of at most 16 unknowns, whose inverse is (1 - A)(1 + A^2)(1 + A^4)(1 + A^8)."""
    case = x["case"]
    n, H, Hk, dk, dv = (case[c] for c in ("n", "H", "Hk", "dk", "dv"))
    count, s, i = _counts(x, n)
    most, dev = case["new_hi"], x["q"].device

    def padded(y):      # [n, heads, tokens, ..] in float32, zeros behind a sequence's last token
        z = torch.zeros(n, most, *y.shape[2:], device=dev)
        z[s, i] = y.flatten(0, 1).float()
        return z.transpose(1, 2)

    q, k, v, g, beta = (padded(x[c]) for c in ("q", "k", "v", "g", "beta"))
    if case["raw"]:
        q, k = (y / torch.sqrt((y * y).sum(-1, keepdim=True) + L2_EPS) for y in (q, k))
        there = (torch.arange(most, device=dev) < count[:, None])[:, None]
        g = torch.where(there, -torch.log1p(torch.exp(g.double())).float(), 0.0)
        beta = torch.where(there, 1 / (1 + torch.exp(-beta)), 0.0)
    q, k = q.repeat_interleave(H // Hk, 1), k.repeat_interleave(H // Hk, 1)
    decay = torch.cumsum(g.double(), -1)
    lower = torch.ones(most, most, device=dev).tril()
    ratio = torch.where(lower > 0, torch.exp(torch.minimum(decay[..., :, None] - decay[..., None, :], decay.new_zeros(()))), 0).float()
    gamma, kt = torch.exp(decay).float()[..., None], k.transpose(2, 3).contiguous()
    A = beta[..., None] * ratio * torch.matmul(k, kt) * lower.tril(-1)
    R = beta[..., None] * (v - gamma * torch.matmul(x["S"], kt).transpose(2, 3))
    A2 = torch.matmul(A, A)
    A4 = torch.matmul(A2, A2)
    U = R + torch.matmul(torch.matmul(A4, A4), R)
    U = U + torch.matmul(A4, U)
    U = U + torch.matmul(A2, U)
    U = U - torch.matmul(A, U)
    out = {}
    if case["outputs"]:
        qs = torch.matmul(x["S"], q.transpose(2, 3).contiguous()).transpose(2, 3)
        o = gamma * qs + torch.matmul(ratio * torch.matmul(q, kt), U)
        out["o"] = o.transpose(1, 2)[s, i].to(x["v"].dtype).view(x["v"].shape)
    if case["keep"] != "none":
        kept = x["keep"].long()
        end = torch.where(kept[:, None] > 0, decay.gather(-1, (kept - 1).clamp(min=0)[:, None, None].expand(-1, H, 1))[..., 0], 0.0)
        part = torch.exp(torch.minimum(end[..., None] - decay, decay.new_zeros(()))).float()
        part = torch.where(torch.arange(most, device=dev) < kept[:, None, None], part, 0.0)
        new = torch.exp(end).float()[..., None, None] * x["S"] + torch.matmul(U.transpose(2, 3).contiguous(), part[..., None] * k)
        x["S"].copy_(torch.where((kept > 0)[:, None, None, None], new, x["S"]))
    out["S"] = x["S"]
    return out


def _plain_verify(x):
    case, p, q = x["case"], x["p"], x["q"]
    n, m, V = case["n"], case["m"], case["V"]
    j, row = torch.arange(m, device=p.device), torch.arange(n, device=p.device)
    lens = torch.full((n,), m, device=p.device) if x["lens"] is None else x["lens"].long().clamp(0, m)
    accepted = torch.zeros_like(lens)
    if m:
        at = x["drafts"].long()[..., None]
        px = p[:, :m].gather(-1, at)[..., 0].double()
        qx = torch.ones_like(px) if q is None else q.gather(-1, at)[..., 0].double()
        taken = (x["u"][:, :m].double() * qx < px) & (j < lens[:, None])
        accepted = torch.cumprod(taken.long(), 1).sum(1)
    target = p[row, accepted].double()
    w = target
    if m:
        stop = accepted.clamp(max=m - 1)
        if q is None:
            less = torch.zeros_like(target).scatter_(1, x["drafts"].long()[row, stop][:, None], 1.0)
        else:
            less = q[row, stop].double()
        w = torch.where((accepted < lens)[:, None], (target - less).clamp(min=0), target)
    w = torch.where(w.sum(-1, keepdim=True) > 0, w, target)
    cdf = torch.cumsum(w, -1)
    found = (cdf <= x["u"][:, m:].double() * cdf[:, -1:]).sum(-1)
    found = torch.minimum(found, (torch.arange(V, device=p.device) * (w > 0)).amax(-1))
    tokens = torch.full((n, m + 1), -1, dtype=torch.int32, device=p.device)
    if m:
        tokens[:, :m] = torch.where(j < accepted[:, None], x["drafts"], -1)
    tokens[row, accepted] = found.int()
    return tokens, (accepted + 1).int()


# ------------------------------------------------------------------ the framework's calls

def _own(x):
    import paper_2607_14568_amd as gdn
    case = x["case"]
    if case["op"] == "tables":
        pool = x["table"], x["held"], x["free"], x["n_free"], case["page"]
        gdn.gdn_cache_tables(x["lens"], *pool, shared=x["shared"], missing=x["missing"], new_lens=x["new_lens"],
                             cu_seqlens=x["cu"], positions=x["positions"], slots=x["slots"])
        gdn.gdn_cache_tables(x["after"], *pool, shared=x["shared"], missing=x["missing"])
        return _tables_out(x)
    if case["op"] == "shared":
        if "workspace" not in x:
            need = gdn.gdn_attention_shared_workspace_bytes(
                *x["q"].shape[:3], case["Hkv"], case["d"], case["page"], x["block_table"].shape[1],
                0 if x["cu"] is None else case["n"], case["groups"])
            x["workspace"] = torch.empty(need, dtype=torch.uint8, device=x["q"].device)
        return gdn.gdn_attention_shared(
            x["q"], x["k_cache"], x["v_cache"], x["block_table"], x["seq_lens"], x["prefix_lens"], cu_groups=x["cu_groups"],
            k_scale=x["k_scale"], v_scale=x["v_scale"], cu_seqlens=x["cu"], o=x["o"], workspace=x["workspace"])
    if case["op"] == "draft":
        flags = gdn.GDN_QK_L2NORM | gdn.GDN_GATE_LOGITS if case["raw"] else 0
        gdn.gdn_draft_step(x["q"] if case["outputs"] else None, x["k"], x["v"], x["g"], x["beta"], x["S"], keep=x["keep"],
                           flags=flags, cu_seqlens=x["cu"], o=x["o"])
        return dict(o=x["o"], S=x["S"]) if case["outputs"] else dict(S=x["S"])
    if "workspace" not in x:
        need = gdn.gdn_draft_verify_workspace_bytes(case["n"], case["m"], case["V"])
        x["workspace"] = torch.empty(need, dtype=torch.uint8, device=x["p"].device)
    return gdn.gdn_draft_verify(x["p"], x["u"], drafts=x["drafts"], q=x["q"], draft_lens=x["lens"], tokens=x["tokens"],
                                counts=x["counts"], workspace=x["workspace"])


def run(state):
    if own:
        return _own(state)
    op = state["case"]["op"]
    if op == "tables":
        _plain_tables(state)
        return _tables_out(state)
    return {"shared": _plain_shared, "draft": _plain_draft, "verify": _plain_verify}[op](state)


def work(case):
    """Inputs read once, outputs written once: the prefix's rows once a group, a state once in and, where tokens are kept, once
    out; of the probabilities one row a sequence and its drafts' own ones."""
    if case["op"] == "tables":
        new, old, after = _sizes(case)
        page, shared = case["page"], case["shared"]
        moved = sum(abs(-(-(a + b) // page) - max(-(-c // page), shared)) for a, b, c in zip(old, new, after))
        return dict(bytes=sum(new) * (4 + 8 + 4) + 2 * (moved * 16 + case["n"] * 16), flops=sum(new) * 4)
    if case["op"] == "shared":
        cuts, prefix, tail, new, empty = _sizes(case)
        H, Hkv, d, page = (case[x] for x in ("H", "Hkv", "d", "page"))
        whole = [p // page * page for p in prefix]
        group = [sum(i >= c for c in cuts[1:]) for i in range(case["n"])]
        rest = [0 if i in empty else prefix[g] - whole[g] + tail[i] for i, g in enumerate(group)]
        keys = sum(whole) + sum(r + (0 if i in empty else new[i]) for i, r in enumerate(rest))
        pairs = sum(0 if i in empty else new[i] * (whole[g] + rest[i]) + new[i] * (new[i] + 1) // 2 for i, g in enumerate(group))
        held = 1 if case["cache"] == "e4m3" else 2
        return dict(bytes=2 * sum(new) * H * d * 2 + keys * 2 * Hkv * (d * held + (0 if held == 2 else 4 / page)), flops=4 * d * H * pairs)
    if case["op"] == "draft":
        new, keep = _sizes(case)
        H, Hk, dk, dv = (case[x] for x in ("H", "Hk", "dk", "dv"))
        size, used = 4 if case["io"] == "f32" else 2, new if case["outputs"] else keep
        states = sum((u > 0) + (a > 0) for u, a in zip(used, keep))
        rows = sum(used) * ((2 * dv * H + 2 * dk * Hk if case["outputs"] else dv * H + dk * Hk) * size + 8 * H)
        return dict(bytes=states * H * dv * dk * 4 + rows, flops=2 * H * dk * dv * ((2 if case["outputs"] else 1) * sum(used) + sum(keep)))
    lens = _sizes(case)
    size, rows = 4 if case["io"] == "f32" else 2, 2 if case["q"] and case["m"] else 1
    return dict(bytes=case["n"] * case["V"] * size * rows + sum(lens) * (2 * size + 12) + case["n"] * 12, flops=case["n"] * case["V"] * 2)


# ------------------------------------------------------------------ exact values

def _exact_shared(case, seed):
    x, (cuts, prefix, tail, new, empty) = _shared_inputs(case, seed), _sizes(case)
    H, Hkv, d, page = (case[c] for c in ("H", "Hkv", "d", "page"))
    q, lens, table, at = x["q"].flatten(0, 1).double(), x["seq_lens"].tolist(), x["block_table"], 0
    out = torch.zeros_like(q)
    for i, a in enumerate(new):
        rows, L = slice(at, at + a), lens[i]
        at += a
        if L == 0:
            continue
        ids = table[i, :-(-L // page)].long()
        hide = torch.arange(L, device=q.device) > torch.arange(L - a, L, device=q.device)[:, None]
        for h in range(Hkv):
            k, v = (x[c + "_cache"][ids, h].double() if x[c + "_scale"] is None else
                    x[c + "_cache"].view(torch.uint8)[ids, h].view(E4M3).double() * x[c + "_scale"][ids, h].double()[:, None, None]
                    for c in "kv")
            k, v = k.reshape(-1, d)[:L], v.reshape(-1, d)[:L]
            heads = slice(h * (H // Hkv), (h + 1) * (H // Hkv))
            score = (q[rows, heads].reshape(-1, d) @ k.t().contiguous()).view(a, -1, L) / math.sqrt(d)
            p = torch.softmax(score.masked_fill(hide[:, None], -math.inf), -1)
            out[rows, heads] = (p.view(-1, L) @ v).view(a, -1, d)
    return out.view(x["q"].shape)


def _exact_draft(case, seed):
    """The recurrence, token by token."""
    x, (new, keep) = _draft_inputs(case, seed), _sizes(case)
    q, k, v, g, beta = (x[c].flatten(0, 1).double() for c in ("q", "k", "v", "g", "beta"))
    if case["raw"]:
        q, k = (y / torch.sqrt(torch.linalg.vector_norm(y, dim=-1, keepdim=True) ** 2 + L2_EPS) for y in (q, k))
        g, beta = torch.log(torch.sigmoid(-g)), torch.sigmoid(beta)
    q, k = (y.repeat_interleave(case["H"] // case["Hk"], 1) for y in (q, k))
    S, o, first = x["S"].double(), torch.zeros_like(v), torch.tensor(_offsets(new)[:-1], device=v.device)
    count, kept = torch.tensor(new, device=v.device), x["keep"].long()
    result = S.clone()
    for j in range(max(new)):
        live = (count > j).nonzero()[:, 0]
        t = first[live] + j
        state = S[live] * torch.exp(g[t])[..., None, None]
        error = v[t] - (state * k[t][:, :, None]).sum(-1)
        state = state + (beta[t][..., None] * error)[..., None] * k[t][:, :, None]
        S[live] = state
        o[t] = (state * q[t][:, :, None]).sum(-1)
        done = kept[live] == j + 1
        result[live[done]] = state[done]
    out = dict(S=result)
    if case["outputs"]:
        out["o"] = o.view(x["v"].shape)
    return out


def exact(case, seed):
    """(The tables and the verification give whole numbers only.)"""
    if case["op"] == "shared":
        return _exact_shared(case, seed)
    return _exact_draft(case, seed) if case["op"] == "draft" else None
