"""Attention over a shared prefix, accumulated weights, eviction and token log
probabilities, written out in numpy float64 for the tests: elementary formulas, no code of
the library; with bounds on how far an fp32 computation may be off."""
import numpy as np

from plain_ops import HALF

EPS = 2.0 ** -24


def prefix_attention(q, k, v, lens, pk, pv, plens, scale=None):
    """q [B, L, Hq, d]; k, v lists of [S_b, Hkv, d]; pk, pv lists of [T_p, Hkv, d].  Row i of
    sequence b sees its whole prefix and own keys j <= S_b - L + i.  Returns o, lse, sum p |v|
    and the largest sum |q k| scale of each row (for bounds)."""
    B, L, Hq, d = q.shape
    n = B // len(pk)
    scale = scale or d ** -0.5
    o, mass = np.zeros((B, L, Hq, d)), np.zeros((B, L, Hq, d))
    lse, qk = np.full((B, L, Hq), -np.inf), np.zeros((B, L, Hq))
    for b in range(B):
        S, T = int(lens[b]), int(plens[b // n])
        kk = np.concatenate([pk[b // n][:T], k[b][:S]])
        vv = np.concatenate([pv[b // n][:T], v[b][:S]])
        G = Hq // kk.shape[1]
        for i in range(L):
            end = T + max(min(S - L + i + 1, S), 0)
            if end == 0:
                continue
            for h in range(Hq):
                x, y = kk[:end, h // G], vv[:end, h // G]
                s = x @ q[b, i, h] * scale
                m = s.max()
                p = np.exp(s - m)
                lse[b, i, h] = m + np.log(p.sum())
                p /= p.sum()
                o[b, i, h] = p @ y
                mass[b, i, h] = p @ np.abs(y)
                qk[b, i, h] = (np.abs(x) @ np.abs(q[b, i, h])).max() * scale
    return o, lse, mass, qk


def prefix_bounds(dtype, n, o, lse, mass, qk, d, vmax):
    """How far o and lse may be off for n keys.  A score: a sum of d products and its scaling in
    the logarithm's base, (d + 8) 2^-24 sum |q k|; a weight by that and the hardware's exp2 (2^-22);
    a sum of n by n 2^-24.  A part's lse: its logarithm, product and sum, 4 2^-24 (|lse| + 2);
    twice that again where the parts meet, and their weights' exp2.  bf16: each weight half a step,
    O half a step.  Weights below 2^-126 of the largest may be lost whole."""
    size = np.abs(np.where(np.isfinite(lse), lse, 0)) + qk + 2
    w = qk * (d + 8) * EPS + 12 * size * EPS + 3 * 2.0 ** -22
    rel = 2 * w + (2 * n + 16) * EPS
    ob = mass * rel[..., None] + np.abs(o) * EPS + n * vmax * 2.0 ** -126
    if dtype == "bf16":
        ob = ob + (mass + np.abs(o)) * HALF["bf16"] * (1 + 2.0 ** -7)
    return ob, w + (n + 16) * EPS


def kv_mass(q, k, lens, lse, mass, pos, pos0, accepted=None, scale=None):
    """k a list of [S_b, Hkv, d].  Returns mass, slot_pos, and a bound on mass's error: a weight by
    its score's (as above), lse's product with log2 e and the sum under the exponential (4 2^-24 (|lse| +
    |s|)), exp2 (2^-22); the sums by a tile's 32 rows and one addition a tile, then the old mass."""
    B, L, Hq, d = q.shape
    Hkv = mass.shape[1]
    G = Hq // Hkv
    scale = scale or d ** -0.5
    mass, pos, err = mass.copy(), pos.copy(), np.zeros(mass.shape)
    for b in range(B):
        S = int(lens[b])
        rows = L if accepted is None else min(max(int(accepted[b]), 0), L - 1) + 1
        base = S - L
        w, e = np.zeros((Hkv, S)), np.zeros((Hkv, S))
        for h in range(Hq):
            kk = k[b][:S, h // G]
            s = q[b, :rows, h] @ kk.T * scale                       # [rows, S]
            z = lse[b, :rows, h][:, None]
            see = np.arange(S)[None] <= base + np.arange(rows)[:, None]
            with np.errstate(invalid="ignore", over="ignore"):
                p = np.where(see & (z > -np.inf), np.exp(s - np.where(z == -np.inf, 0, z)), 0.0)
            size = (np.abs(q[b, :rows, h]) @ np.abs(kk).T) * scale
            zs = np.where(np.isfinite(z), np.abs(z), 0)
            w[h // G] += p.sum(0)
            e[h // G] += (p * (size * (d + 12) * EPS + 4 * zs * EPS + 2.0 ** -21)).sum(0)
        e += w * (rows * G / 32 + 16) * EPS
        new = np.arange(S) >= base
        mass[b, :, :S] = np.where(new, w, mass[b, :, :S] + w)
        err[b, :, :S] = e + np.abs(mass[b, :, :S]) * EPS * 1.01 + rows * G * 2.0 ** -126
        for j in range(max(base, 0), S):
            pos[b, :, j] = pos0[b] + j - base
    return mass, pos, err


def evict(rows, mass, pos, lens, seq, budget, n_sink, recent):
    """rows [B, Hkv, slots]: what each slot holds (any array).  Returns the same after the call,
    mass, pos and lengths."""
    rows, mass, pos = rows.copy(), mass.copy(), pos.copy()
    B, Hkv, slots = mass.shape
    for b in range(B):
        n = min(max(int(lens[b]), 0), slots)
        if n <= budget:
            continue
        for h in range(Hkv):
            m, x = mass[b, h, :n].astype(np.float64), pos[b, h, :n]
            held = (x < n_sink) | (x >= int(seq[b]) - recent)
            # Held tokens last, among themselves by slot; NaN below -inf.
            order = sorted(range(n), key=lambda j: (1, 0, 0, j) if held[j] else
                           (0, not np.isnan(m[j]), 0 if np.isnan(m[j]) else m[j], j))
            out = set(order[: n - budget])
            holes = [j for j in range(budget) if j in out]
            kept = [j for j in range(budget, n) if j not in out]
            assert len(holes) == len(kept)
            for to, src in zip(holes, kept):
                for t in (rows, mass, pos):
                    t[b, h, to] = t[b, h, src]
    return rows, mass, pos, np.minimum(np.clip(lens, 0, slots), budget)


def token_logprobs(x, tokens, top_k):
    """x [rows, V].  Returns logprobs, entropy, top, top_logprobs and the sum's logarithm (ln z)."""
    n, V = x.shape
    lp, ent, lz = np.zeros(n), np.zeros(n), np.zeros(n)
    top, tlp = np.full((n, top_k), -1), np.full((n, top_k), -np.inf)
    for r in range(n):
        bad = np.isnan(x[r]).any() or (x[r] == np.inf).any()
        m = x[r].max()
        if bad:
            lse, ent[r] = np.nan, np.nan
        elif m == -np.inf:
            lse, ent[r] = -np.inf, 0.0
        else:
            p = np.exp(x[r] - m)
            z = p.sum()
            lse, lz[r] = m + np.log(z), np.log(z)
            q = p / z
            ent[r] = -(q[q > 0] * np.log(q[q > 0])).sum()

        def of(v):
            return np.nan if bad else (-np.inf if v == -np.inf else v - lse)
        if tokens is not None and tokens[r] >= 0:
            lp[r] = of(x[r, tokens[r]]) if tokens[r] < V else np.nan
        order = np.argsort(-np.where(np.isnan(x[r]), -np.inf, x[r]), kind="stable")[:top_k]
        top[r, : len(order)] = order
        tlp[r, : len(order)] = [of(v) for v in x[r][order]]
    return lp, ent, top, tlp, lz


def logprob_bound(lp, lse_size, chunks=1):
    """A weight exp(x - m): the difference, its product with log2 e and exp2, 8 2^-24 (|d| e^-|d| < 1);
    sums of 16 and 4, then 8 of joins of at most 16, each an exp2 and two roundings (8 2^-24), and as
    many again where segments meet; the logarithm and the last difference."""
    return (8 + 24 + 16 * (16 + chunks)) * EPS + 4 * EPS * (np.abs(lse_size) + np.abs(lp) + 1)
