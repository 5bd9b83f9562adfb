"""Inputs of gdn_draft_step's tests, and how far its fp32 steps may be from the recurrence in 64 bits, counted rounding by rounding."""
import numpy as np
import torch

import oracle
from oracle.paged import spans

IO = {"bf16": torch.bfloat16, "f32": torch.float32}
TILE = 8
bf16 = lambda x: torch.from_numpy(np.asarray(x)).bfloat16().double().numpy()   # noqa: E731


def make(seed, rows, n, H, Hk, dk, dv, io, raw):
    """q, k, v, g, beta and the states on the CPU: unit q and k, gates of 0 to 1; ``raw``: q and k of any length, logits."""
    r = np.random.default_rng(seed)
    t = lambda *s: torch.from_numpy(r.standard_normal(s))   # noqa: E731
    q, k, v, a, b, S = t(*rows, Hk, dk), t(*rows, Hk, dk), t(*rows, H, dv), t(*rows, H), t(*rows, H), 0.3 * t(n, H, dv, dk)
    if not raw:
        q, k = (x / x.norm(dim=-1, keepdim=True) for x in (q, k))
        a, b = -torch.nn.functional.softplus(a - 1), torch.sigmoid(b)
    return [x.to(IO[io]) for x in (q, k, v)] + [x.float() for x in (a, b, S)]


def walk(q, k, v, g, beta, S, keep, cu, raw, scale, wrong=None):
    """(o, S after the kept tokens, bounds of both) from values in 64 bits, tile by tile as the kernel goes; ``wrong`` names a mistake.

    Roundings (e = 2^-24 of a partial sum, signs of their own; n of size a_j add up to more than 8 (sum a_j^2)^1/2 with a
    probability under 2 exp(-32)).  A token's update c_t = beta (v - gamma S k_t - sum c_i k_i.k_t), of each state row:
      S k_t: dk of at most e |S|;  each k_i.k_t: dk of at most e, times c_i;  the 2 (8 + 4) sums and decays: of at most e times
      |v| + gamma |S k_t| + sum |c_i k_i.k_t|
    and the state's update 8 + 1 of at most e (|S| + sum |c_i|) an element (times dk^1/2 for the row).  What a token's update is
    off by moves the state by as much along k_t and passes the later tokens' (1 - beta k k^T) alpha without growing; an output
    is scale q times the state, with its own dk of e |S| and those of its pairs.
    Not of signs of their own: decays, gates and norms by the library's functions, 2^-22 of themselves each (with logits 2 + |g|
    times that), of |S| + |c| a token; the rows' lengths 2^-8 off 1 in bf16 are covered by taking |k|^2 <= 1.02 below."""
    q, k, v, g, beta, S = (np.array(y, dtype=np.float64) for y in (q, k, v, g, beta, S))
    if wrong == "bf16 inputs":
        q, k, S = bf16(q), bf16(k), bf16(S)
    if raw:
        q, k = oracle.l2_rows(q), oracle.l2_rows(k)
        g, beta = oracle.gates_from_logits(g, beta)
    if wrong == "gates":
        g = g * 1.01
    if wrong == "beta":
        beta = beta * 0.99
    B, T, H, dv = v.shape
    G, dk, e = H // k.shape[2], k.shape[3], 2.0 ** -24
    q, k, v, g, beta = (y.reshape(B * T, *y.shape[2:]) for y in (q, k, v, g, beta))
    q, k = (np.repeat(y, G, 1) for y in (q, k))
    o, off_o = np.full(v.shape, np.nan), np.full(v.shape, np.nan)
    kept_S, off_S = S.copy(), np.zeros(S.shape[:3])
    for s, (at, m) in enumerate(spans(B, T, cu)):
        kept = m if keep is None else min(max(int(keep[s]), 0), m)
        state, var, drift = S[s], np.zeros((H, dv)), np.zeros((H, dv))
        for t0 in range(0, m, TILE):
            if wrong == "bf16 between tiles" and t0:
                state = bf16(state)
            size = np.linalg.norm(state, axis=-1)
            c, gamma, ks = [], np.ones(H), []
            for t in range(at + t0, at + min(t0 + TILE, m)):
                alpha = np.exp(g[t])
                gamma = gamma * alpha
                x = gamma[:, None] * np.einsum("hvk,hk->hv", state, k[t])
                c = [alpha[:, None] * y for y in c]
                pairs = [y * (z * k[t]).sum(-1)[:, None] for y, z in zip(c, ks)]
                new = beta[t][:, None] * (v[t] - x - (0 if wrong == "pairs" else sum(pairs)))
                terms = np.abs(v[t]) + np.abs(x) + sum(np.abs(y) for y in pairs)
                var = var + e * e * (dk * (size ** 2 + sum(y * y for y in c)) + 24 * terms ** 2)
                c, ks = c + [new], ks + [k[t]]
                far = (2 + np.abs(g[t]) if raw else np.ones(H))[:, None]
                drift = drift + 2.0 ** -22 * far * (size + np.abs(new))
                now = gamma[:, None, None] * state + sum(y[..., None] * z[:, None] for y, z in zip(c, ks))
                o[t] = scale * (gamma[:, None] * np.einsum("hvk,hk->hv", state, q[t]) + sum(y * (z * q[t]).sum(-1)[:, None] for y, z in zip(c, ks)))
                mine = e * e * (dk * (size ** 2 + sum(y * y for y in c)) + 24 * (size + sum(np.abs(y) for y in c)) ** 2)
                off_o[t] = scale * (8 * np.sqrt(1.02 * (var + mine)) + drift + 2.0 ** -22 * size)
                if t - at + 1 == kept:
                    put = 9 * dk * e * e * (size + sum(np.abs(y) for y in c)) ** 2
                    kept_S[s], off_S[s] = now, 8 * np.sqrt(1.02 * (var + put / dk)) + drift
            var = var + 9 * e * e * (size + sum(np.abs(y) for y in c)) ** 2
            state = now
    return o.reshape(B, T, H, dv), kept_S, off_o.reshape(B, T, H, dv), off_S[..., None]


def worst(got_o, got_S, ref, io):
    """The largest error of outputs (None: none) and states over their bounds; outputs are rounded once to ``io``."""
    o, S, off_o, off_S = ref
    most = (np.abs(got_S - S) / (off_S + 2.0 ** -24 * np.abs(S) + 1e-30)).max()
    if got_o is None:
        return most
    live = ~np.isnan(o)
    half = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}[io]
    return max(most, (np.abs(got_o - o)[live] / (off_o + half * np.abs(o) + 1e-30)[live]).max(initial=0.0))
