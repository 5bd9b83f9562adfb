"""The attention layers' serving operators: what is measured, their plain forms, and exact values to hold both against.

Three operators of the backbone's attention layers:

  norm       RMS norm of the queries and keys of each head and the position rotation, in one pass over a prompt's q and k
  append     the new tokens' keys and values into a paged cache (bfloat16, or e4m3 with one scale per page and head), keys
             normed and rotated on the way, queries transformed in the same pass
  attention  the new tokens' attention over that cache: one token a sequence, a few, or a long piece of a prompt

A step of a sequence brings ``new`` tokens to ``old`` ones; all its calls share ``seq_lens`` (old + new), the block table and
the packed offsets.  ``listed()`` names twelve cases, ``draw(rng)`` gives others of the same ranges: 1 to 256 sequences, 1 to
10240 new tokens, up to 131072 in the cache, 8 to 32 query heads over 2 to 16 key/value heads of 64 or 128, pages of 16 to
128 tokens, rotated widths of 16 to the head's.

Cache pages are [n_pages, H_kv, page, d], their scales [n_pages, H_kv] (float32, a power of two: the smallest s with every
finite value of the page's head at most 448 s).  What is held in 8 bits is returned as float8 values beside its scales.
"""
from __future__ import annotations

import math
import random

import torch

own = False

EPS = 1e-6
E4M3 = torch.float8_e4m3fn
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": E4M3}


def _case(name, op, n, new, old=(0, 0), *, H=16, Hkv=8, d=128, rot=None, io="bf16", cache="bf16", page=64, pairs="half",
          norm=True, wide=False, mix=0):
    """``new``, ``old``: the ranges that the sequences' lengths are spread over.  ``wide``: q, k and v are parts of one
    projection's rows.  ``pairs``: which channels rotate together, a half apart or next to each other."""
    return dict(name=name, op=op, n=n, new_lo=new[0], new_hi=new[1], old_lo=old[0], old_hi=old[1], H=H, Hkv=Hkv, d=d,
                rot=d if rot is None else rot, io=io, cache=cache, page=page, pairs=pairs, norm=norm, wide=wide, mix=mix)


def listed():
    return [
        # the long prompt of the library's main workload, ahead of its causal attention
        _case("norm_prompt_bf16", "norm", 1, (10240, 10240)),
        # packed prompts of a serving batch: small heads, half of each rotated, rows of a fused projection
        _case("norm_packed_bf16", "norm", 8, (60, 2900), Hkv=4, d=64, rot=32, wide=True, mix=1),
        # one user's next token: latency
        _case("append_b1_bf16", "append", 1, (1, 1), (2000, 2000), wide=True),
        # the next token of a large serving batch into an 8-bit cache, pages partly filled
        _case("append_b256_e4m3", "append", 256, (1, 1), (16, 2048), cache="e4m3", wide=True, mix=2),
        # packed pieces of prompts behind what the cache holds of them
        _case("append_packed_bf16", "append", 8, (512, 4096), (0, 4000), page=32, mix=3, wide=True),
        # an odd prompt into an 8-bit cache
        _case("append_prompt_e4m3", "append", 1, (4133, 4133), (1000, 1000), cache="e4m3"),
        # one user's next token after a short exchange: latency
        _case("attention_b1_bf16", "attention", 1, (1, 1), (776, 776)),
        # a serving batch's next token, lengths a factor of sixteen apart
        _case("attention_b64_bf16", "attention", 64, (1, 1), (512, 8191), mix=4),
        # the same from an 8-bit cache
        _case("attention_b64_e4m3", "attention", 64, (1, 1), (512, 8191), cache="e4m3", mix=4),
        # one user's next token after a very long document: the cache's length is split
        _case("attention_long_bf16", "attention", 1, (1, 1), (131071, 131071)),
        # four drafted tokens a sequence to verify, four query heads a key/value head
        _case("attention_draft_e4m3", "attention", 16, (4, 4), (100, 16384), Hkv=4, cache="e4m3", page=16, mix=5),
        # a piece of a long prompt behind the part already in the cache
        _case("attention_piece_bf16", "attention", 1, (2048, 2048), (8192, 8192)),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(max(1, lo)), math.log(max(1, hi))))))


def draw(rng):
    op = rng.choice(["norm", "append", "append", "attention", "attention", "attention"])
    H, d = rng.choice([8, 16, 16, 32]), rng.choice([64, 128, 128])
    Hkv = rng.choice([h for h in (2, 4, 8, 16) if h <= H])
    rot = rng.choice([16, d // 4, d // 2, d, d])
    kw = dict(H=H, Hkv=Hkv, d=d, rot=rot, page=rng.choice([16, 32, 64, 64, 128]), cache=rng.choice(["bf16", "e4m3"]),
              pairs=rng.choice(["half", "half", "near"]), norm=rng.random() < 0.8, wide=rng.random() < 0.5,
              mix=rng.randrange(1000))
    row = 16 * 128 / (H * d)                     # a case's tokens, by what one of its rows holds
    if op == "norm":
        n = rng.randint(1, 8)
        hi = max(64, int(10240 * min(1, row)) // n)
        io = rng.choice(["bf16", "bf16", "f32"])
        top = _log_int(rng, 64, hi if io == "bf16" else max(64, hi // 2))
        c = _case("", "norm", n, (max(1, top // rng.choice([1, 4, 40])), top), io=io, **kw)
    elif op == "append":
        if rng.random() < 0.5:
            c = _case("", "append", _log_int(rng, 1, 256), (1, 1), (rng.randint(0, 16), _log_int(rng, 16, 2048)), **kw)
        else:
            n = rng.randint(1, 8)
            top = _log_int(rng, 8, max(8, int(10240 * min(1, row)) // n))
            c = _case("", "append", n, (max(1, top // rng.choice([1, 4, 40])), top), (0, _log_int(rng, 16, 4096)), **kw)
    else:
        keys = 177000 * 1024 // (Hkv * d)        # cached tokens of a call, over all its sequences
        form = rng.choice(["batch", "batch", "long", "draft", "piece"])
        if form == "long":
            top = _log_int(rng, 8192, min(131072, keys))
            c = _case("", "attention", 1, (1, 1), (top, top), **kw)
        elif form == "piece":
            n = rng.randint(1, 4)
            top = _log_int(rng, 17, max(17, int(2048 * min(1, row)) // n))
            c = _case("", "attention", n, (max(1, top // rng.choice([1, 4])), top), (0, _log_int(rng, 16, 8192)), **kw)
        else:
            n = _log_int(rng, 1, 128)
            new = 1 if form == "batch" else rng.randint(2, 8)
            top = max(16, min(16384, keys // n))
            lo = max(0, top // rng.choice([1, 4, 16]))
            c = _case("", "attention", n, (new, new), (lo, _log_int(rng, max(1, lo), top)), **kw)
    del c["name"]
    return c


def _lengths(case):
    """(new, old) of every sequence, spread over the logarithm of their ranges."""
    rng = random.Random(case["mix"])
    new = [_log_int(rng, case["new_lo"], case["new_hi"]) for _ in range(case["n"])]
    old = [_log_int(rng, case["old_lo"] + 1, case["old_hi"] + 1) - 1 for _ in range(case["n"])]
    return new, old


def _dense(case):
    return case["new_lo"] == case["new_hi"]


def _inputs(case, seed):
    """The call's inputs on the GPU, from the seed alone."""
    dev = torch.device("cuda", torch.cuda.current_device())
    rng = torch.Generator(device=dev)
    rng.manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=rng, device=dev, dtype=torch.float32)

    def ints(values):
        return torch.tensor(values, dtype=torch.int32).to(dev)

    new, old = _lengths(case)
    n, H, Hkv, d, page, io = (case[x] for x in ("n", "H", "Hkv", "d", "page", "io"))
    rows = (n, new[0]) if _dense(case) else (1, sum(new))
    x = dict(case=case, cu=None if _dense(case) else ints([sum(new[:i]) for i in range(n + 1)]))
    heads = dict(q=H) if case["op"] == "attention" else dict(q=H, k=Hkv) if case["op"] == "norm" else dict(q=H, k=Hkv, v=Hkv)
    if case["wide"] and case["op"] != "attention":
        every = normal(*rows, sum(heads.values()), d).to(DTYPES[io])
        x.update(zip(heads, every.split(list(heads.values()), dim=2)))
    else:
        x.update((name, normal(*rows, h, d).to(DTYPES[io])) for name, h in heads.items())
    if case["op"] != "attention":
        x["inv_freq"] = 10000.0 ** (-torch.arange(0, case["rot"], 2, dtype=torch.float64) / case["rot"]).to(dev)
        x["q_weight"] = 1 + 0.1 * normal(d) if case["norm"] else None
        x["k_weight"] = 1 + 0.1 * normal(d) if case["norm"] else None
    if case["op"] == "norm":
        return x
    # the cache: a page for every started block of every sequence, and a few more, in an order of its own
    need = [-(-(a + b) // page) for a, b in zip(new, old)]
    n_pages, width = sum(need) + 3, max(need) + 1
    order = torch.randperm(n_pages, generator=rng, device=dev).to(torch.int32)
    first = [sum(need[:i]) for i in range(n)]
    at = torch.tensor(first)[:, None] + torch.arange(width)
    held = torch.arange(width) < torch.tensor(need)[:, None]
    x["block_table"] = torch.where(held.to(dev), order[at.clamp(max=n_pages - 1).to(dev)], order.new_full((), -1))
    x["seq_lens"] = ints([a + b for a, b in zip(new, old)])
    for name in ("k", "v"):
        size = torch.exp(0.5 * normal(n_pages, Hkv))
        values = normal(n_pages, Hkv, page, d)
        if case["cache"] == "bf16":
            x[name + "_cache"], x[name + "_scale"] = values.bfloat16(), None
        else:   # values of about unit size, each page and head with a size of its own
            scale = torch.exp2(torch.floor(torch.log2(size)) - 6)
            x[name + "_cache"] = (values * size[..., None, None] / scale[..., None, None]).clamp(-448, 448).to(E4M3)
            x[name + "_scale"] = scale
    return x


def prepare(case, seed):
    """Inputs, the cache, and the output buffer that a serving program keeps."""
    x = _inputs(case, seed)
    x["q_out"] = torch.empty(x["q"].shape, dtype=x["q"].dtype, device=x["q"].device)
    if case["op"] == "norm":
        x["k_out"] = torch.empty(x["k"].shape, dtype=x["k"].dtype, device=x["k"].device)
    return x


# ------------------------------------------------------------------ the plain forms

def _tokens(x):
    """Of every token of the call: its sequence, its place among the sequence's new tokens, and how many these are."""
    B, T = x["q"].shape[:2]
    t = torch.arange(B * T, device=x["q"].device)
    if x["cu"] is None:
        return t // T, t % T, torch.full_like(t, T)
    cu = x["cu"].long()
    s = (t[:, None] >= cu[1:]).sum(1)
    return s, t - cu[s], cu[s + 1] - cu[s]


def _turned(x, name, pos):
    """The normed and rotated rows of x[name] in float32, [tokens, heads, d]; angles in float64."""
    case, y, w = x["case"], x[name].flatten(0, 1).float(), x[name + "_weight"]
    if w is not None:
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * w
    angle = (pos.double()[:, None] * x["inv_freq"])[:, None, :]
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    r = case["rot"]
    if case["pairs"] == "half":
        a, b = y[..., :r // 2], y[..., r // 2:r]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = y[..., 0:r:2], y[..., 1:r:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([turned, y[..., r:]], -1)


def _power_scale(largest):
    """The smallest power of two, at least 2^-100, with largest <= 448 s."""
    m, e = torch.frexp(largest)                                    # largest = m 2^e, 1/2 <= m < 1; 448 = 0.875 2^9
    return torch.exp2(torch.where(largest > 0, e - 9 + (m > 0.875), -100).clamp(min=-100).float())


def _append_e4m3(x, name, rows, s, page_id, slot):
    """``rows`` [tokens, H_kv, d] into the 8-bit cache: scales of the touched pages, the codes that were in a sequence's first
    page brought to its new scale, then the new codes."""
    cache, scale, case = x[name + "_cache"], x[name + "_scale"], x["case"]
    n_pages, Hkv = scale.shape
    most = torch.zeros_like(scale).scatter_reduce_(0, page_id[:, None].expand(-1, Hkv), rows.abs().amax(-1), "amax")
    first = x["seq_lens"].long() - _counts(x)                      # every sequence's first new position
    touched = x["block_table"].long().gather(1, (first // case["page"])[:, None])[:, 0]
    held = first % case["page"]                                    # tokens that this page held
    before = scale[touched]
    fresh = _power_scale(most)
    after = torch.where(held[:, None] > 0, torch.maximum(before, fresh[touched]), fresh[touched])
    codes = cache.view(torch.uint8)                                # (which torch moves by index)
    old = codes[touched].view(E4M3).float()
    keep = (torch.arange(case["page"], device=held.device) < held[:, None])[:, None, :, None]
    codes[touched] = torch.where(keep, old * (before / after)[..., None, None], old).to(E4M3).view(torch.uint8)
    scale[page_id] = fresh[page_id]
    scale[touched] = after
    codes[page_id, :, slot] = (rows / scale[page_id][..., None]).to(E4M3).view(torch.uint8)


def _counts(x):
    if x["cu"] is None:
        return torch.full_like(x["seq_lens"], x["q"].shape[1]).long()
    return (x["cu"][1:] - x["cu"][:-1]).long()


def _plain_norm(x):
    _, i, _ = _tokens(x)
    return [_turned(x, name, i).to(x[name].dtype).view(x[name].shape) for name in ("q", "k")]


def _plain_append(x):
    s, i, n = _tokens(x)
    pos = x["seq_lens"].long()[s] - n + i
    page_id = x["block_table"].long()[s, pos // x["case"]["page"]]
    slot = pos % x["case"]["page"]
    k, v = _turned(x, "k", pos), x["v"].flatten(0, 1).float()
    for name, rows in (("k", k), ("v", v)):
        if x["case"]["cache"] == "e4m3":
            _append_e4m3(x, name, rows, s, page_id, slot)
        else:
            x[name + "_cache"][page_id, :, slot] = rows.bfloat16()
    out = [_turned(x, "q", pos).bfloat16().view(x["q"].shape), x["k_cache"], x["v_cache"]]
    return out + [x["k_scale"], x["v_scale"]] if x["case"]["cache"] == "e4m3" else out


def _gathered(x, name):
    """The sequences' keys or values in float32, [n, H_kv, pages * page, d]."""
    ids = x["block_table"].long().clamp(min=0)
    y = x[name + "_cache"]
    y = (y.view(torch.uint8)[ids].view(E4M3) if y.dtype == E4M3 else y[ids]).float()     # [n, pages, H_kv, page, d]
    if x[name + "_scale"] is not None:
        y = y * x[name + "_scale"][ids][..., None, None]
    return y.transpose(1, 2).flatten(2, 3)


def _plain_attention(x):
    case = x["case"]
    n, H, Hkv, d = (case[c] for c in ("n", "H", "Hkv", "d"))
    s, i, count = _tokens(x)
    most = case["new_hi"]
    q = torch.zeros(n, most, H, d, device=x["q"].device)
    q[s, i] = x["q"].flatten(0, 1).float()
    q = q.view(n, most, Hkv, H // Hkv, d).permute(0, 2, 1, 3, 4).flatten(2, 3)           # [n, H_kv, rows, d]
    k, v = _gathered(x, "k"), _gathered(x, "v")
    score = torch.matmul(q, k.transpose(2, 3).contiguous()) / math.sqrt(d)
    last = (x["seq_lens"].long() - _counts(x))[:, None] + torch.arange(most, device=q.device)
    key = torch.arange(k.shape[2], device=q.device)
    seen = (key <= last[..., None]).repeat_interleave(H // Hkv, 1)[:, None]
    score = torch.where(seen, score, score.new_full((), -math.inf))
    p = torch.exp(score - score.amax(-1, keepdim=True))
    o = torch.matmul(p, v) / p.sum(-1, keepdim=True)
    o = o.view(n, Hkv, most, H // Hkv, d).permute(0, 2, 1, 3, 4).flatten(2, 3)           # [n, rows, H, d]
    return o[s, i].bfloat16().view(x["q"].shape)


# ------------------------------------------------------------------ the framework's calls

def _own(x):
    import paper_2607_14568_amd as gdn
    case = x["case"]
    turn = {c: x.get(c) for c in ("q_weight", "k_weight", "inv_freq")}
    turn.update(eps=EPS, interleaved=case["pairs"] == "near", q_out=x["q_out"], cu_seqlens=x["cu"])
    if case["op"] == "norm":
        return gdn.gdn_qk_norm_rope(x["q"], x["k"], k_out=x["k_out"], **turn)
    cache = x["k_cache"], x["v_cache"], x["block_table"], x["seq_lens"]
    scales = dict(k_scale=x["k_scale"], v_scale=x["v_scale"])
    if case["op"] == "append":
        q = gdn.gdn_kv_append(x["k"], x["v"], *cache, q=x["q"], **scales, **turn)
        out = [q, x["k_cache"], x["v_cache"]]
        return out + [x["k_scale"], x["v_scale"]] if case["cache"] == "e4m3" else out
    if "workspace" not in x:   # what a serving program keeps from step to step
        need = gdn.gdn_attention_paged_workspace_bytes(
            *x["q"].shape[:3], case["Hkv"], case["d"], case["page"], x["block_table"].shape[1],
            0 if x["cu"] is None else case["n"])
        x["workspace"] = torch.empty(need, dtype=torch.uint8, device=x["q"].device)
    return gdn.gdn_attention_paged(x["q"], *cache, cu_seqlens=x["cu"], o=x["q_out"], workspace=x["workspace"], **scales)


def run(state):
    if own:
        return _own(state)
    return {"norm": _plain_norm, "append": _plain_append, "attention": _plain_attention}[state["case"]["op"]](state)


def work(case):
    """Every input row read once, every output row written once; the cached rows that the step's queries see, once."""
    new, old = _lengths(case)
    H, Hkv, d = case["H"], case["Hkv"], case["d"]
    size = 4 if case["io"] == "f32" else 2
    held = 1 if case["cache"] == "e4m3" else 2
    tokens = sum(new)
    if case["op"] == "norm":
        return dict(bytes=2 * tokens * (H + Hkv) * d * size, flops=tokens * (H + Hkv) * d * 8)
    if case["op"] == "append":
        pages = sum(-(-(a + b) // case["page"]) - b // case["page"] for a, b in zip(new, old))
        scales = 0 if held == 2 else 2 * 4 * pages * Hkv
        return dict(bytes=tokens * ((2 * H + 2 * Hkv) * 2 + 2 * Hkv * held) * d + scales, flops=tokens * (H + Hkv) * d * 8)
    pairs = sum(a * b + a * (a + 1) // 2 for a, b in zip(new, old))
    scales = 0 if held == 2 else 2 * 4 * Hkv * sum(-(-(a + b) // case["page"]) for a, b in zip(new, old))
    return dict(bytes=2 * tokens * H * d * 2 + sum(a + b for a, b in zip(new, old)) * 2 * Hkv * d * held + scales,
                flops=4 * d * H * pairs)


# ------------------------------------------------------------------ exact values

def _e4m3(y):
    """The nearest e4m3 value (ties to even), in float64: three bits behind the leading one, steps of 2^-9 below 2^-6."""
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step


def _exact_rows(case, x, name, start):
    """One sequence's rows x[name] (float64 [T, heads, d]) normed and rotated, their first position ``start``."""
    y, out, r = x[name], x[name].clone(), case["rot"]
    if x[name + "_weight"] is not None:
        y = y / torch.sqrt(torch.linalg.vector_norm(y, dim=-1, keepdim=True) ** 2 / case["d"] + EPS)
        y = y * x[name + "_weight"].double()
        out = y.clone()
    pos = torch.arange(start, start + y.shape[0], device=y.device, dtype=torch.float64)
    z = torch.polar(torch.ones((), device=y.device, dtype=torch.float64), torch.outer(pos, x["inv_freq"]))[:, None]
    a, b = (slice(0, r // 2), slice(r // 2, r)) if case["pairs"] == "half" else (slice(0, r, 2), slice(1, r, 2))
    w = torch.complex(y[..., a].contiguous(), y[..., b].contiguous()) * z
    out[..., a], out[..., b] = w.real, w.imag
    return out


def _exact_append(case, x, name, rows, table, start):
    """One sequence's rows [T, H_kv, d] (float64) into the float64 images of the cache and its scales, page by page."""
    cache, scale, page = x[name + "_cache"], x[name + "_scale"], case["page"]
    at = 0
    while at < rows.shape[0]:
        p, slot = divmod(start + at, page)
        part = rows[at:at + page - slot].transpose(0, 1)           # [H_kv, tokens, d]
        i, many = table[p], part.shape[1]
        if scale is not None:
            s = torch.exp2(torch.ceil(torch.log2(part.abs().amax((1, 2)) / 448)).clamp(min=-100))
            if slot:
                s = torch.maximum(s, scale[i])
                cache[i, :, :slot] = _e4m3(cache[i, :, :slot] * (scale[i] / s)[:, None, None])
            scale[i] = s
            part = _e4m3(part / s[:, None, None])
        cache[i, :, slot:slot + many] = part
        at += many


def exact(case, seed):
    x = _inputs(case, seed)
    new, old = _lengths(case)
    H, Hkv, d, op = case["H"], case["Hkv"], case["d"], case["op"]
    names = [c for c in ("q", "k", "v") if c in x]
    shape = {c: x[c].shape for c in names}
    whole = {c: x[c].flatten(0, 1).double() for c in names}
    out = {c: torch.empty_like(whole[c]) for c in names}
    if op == "append":
        for c in ("k_cache", "v_cache", "k_scale", "v_scale"):
            x[c] = x[c].double() if x[c] is not None else None
    if op != "norm":
        tables = x["block_table"].tolist()
    at = 0
    for i, (a, b) in enumerate(zip(new, old)):
        span = slice(at, at + a)
        at += a
        part = dict(x, **{c: whole[c][span] for c in names})
        if op == "norm":
            for c in names:
                out[c][span] = _exact_rows(case, part, c, 0)
        elif op == "append":
            out["q"][span] = _exact_rows(case, part, "q", b)
            _exact_append(case, x, "k", _exact_rows(case, part, "k", b), tables[i], b)
            _exact_append(case, x, "v", part["v"], tables[i], b)
        else:
            ids = torch.tensor(tables[i][:-(-(a + b) // case["page"])], device=part["q"].device)
            for h in range(Hkv):
                k, v = (x[c + "_cache"][:, h].float()[ids].double() * (1 if x[c + "_scale"] is None else
                                                              x[c + "_scale"][ids, h].double()[:, None, None]) for c in "kv")
                k, v = (t.reshape(-1, d)[:a + b].contiguous() for t in (k, v))
                for lo in range(0, a, 512):
                    part_q = part["q"][lo:lo + 512, h * (H // Hkv):(h + 1) * (H // Hkv)]
                    for g in range(H // Hkv):
                        score = part_q[:, g].contiguous() @ k.t().contiguous() * d ** -0.5
                        hide = torch.arange(a + b, device=k.device) > \
                            torch.arange(b + lo, b + lo + score.shape[0], device=k.device)[:, None]
                        out["q"][at - a + lo:at - a + lo + score.shape[0], h * (H // Hkv) + g] = \
                            torch.softmax(score.masked_fill(hide, -math.inf), 1) @ v
    if op == "attention":
        return out["q"].view(shape["q"])
    if op == "norm":
        return [out[c].view(shape[c]) for c in ("q", "k")]
    back = [out["q"].view(shape["q"]), x["k_cache"], x["v_cache"]]
    return back + [x["k_scale"], x["v_scale"]] if case["cache"] == "e4m3" else back
