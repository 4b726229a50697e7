"""The 4-bit cache's format, its attention, sampled acceptance and the query/key norm
with rotation, written out in numpy float64 for the tests: elementary loops and
formulas, no code of the library."""
import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])

# Half a step relative to the value, and the same of fp32.
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def kv4_round(x):
    """x [..., d] -> (codes [..., d] 0..15, scale bytes [..., d / 32])."""
    x = np.asarray(x, np.float64)
    blk = x.reshape(x.shape[:-1] + (-1, 32))
    a = np.abs(blk).max(-1)
    bad = ~np.isfinite(blk).all(-1)
    m, ex = np.frexp(np.where(bad, 0.0, a))      # a = m 2^ex, 0.5 <= m < 1
    e = np.where(m >= 0.875, ex - 2, ex - 3)     # floor(log2(8 a / 7)) - 2
    e = np.clip(np.where(a == 0, -125, e), -125, 125)
    with np.errstate(invalid="ignore"):
        y = np.abs(blk) / np.exp2(e.astype(np.float64))[..., None]
    codes = np.zeros(y.shape, np.int64)
    for k in range(7):                           # from level k to k + 1 past the midpoint
        mid = (LEVELS[k] + LEVELS[k + 1]) / 2
        codes += (y > mid) | ((y == mid) & (k % 2 == 1))
    codes += 8 * np.signbit(blk)
    codes[bad] = 0
    return codes.reshape(x.shape), np.where(bad, 255, e + 127).astype(np.int64)


def kv4_values(codes, scales):
    s = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    v = np.where(codes >= 8, -1.0, 1.0) * LEVELS[codes & 7] * np.repeat(s, 32, -1)
    # bf16 and fp32 end below 2^128, which codes under the scales 253 and 254 can reach.
    return np.where(np.abs(v) >= 2.0 ** 128, np.copysign(np.inf, v), v)


def pack(codes):
    return (codes[..., 0::2] | (codes[..., 1::2] << 4)).astype(np.uint8)


def unpack(b):
    b = b.astype(np.int64)
    return np.stack([b & 15, b >> 4], -1).reshape(b.shape[:-1] + (-1,))


def attention(q, k, v, lens, n_sink=0, window=None, scale=None):
    """q [B, L, Hq, d]; k, v lists of [S_b, Hkv, d] in token order.  Returns o, lse, and
    sum p |v| (for error bounds), sum |q k| scale at its largest."""
    B, L, Hq, d = q.shape
    o = np.zeros((B, L, Hq, d))
    mass, lse, qk = np.zeros((B, L, Hq, d)), np.full((B, L, Hq), -np.inf), np.zeros((B, L, Hq))
    scale = scale or d ** -0.5
    for b in range(B):
        S = int(lens[b])
        Hkv = k[b].shape[1]
        for i in range(L):
            pos = S - L + i
            j = np.arange(max(pos + 1, 0))
            if window is not None:
                j = j[(j < n_sink) | (j > pos - window)]
            if not len(j):
                continue
            for h in range(Hq):
                kk, vv = k[b][j, h // (Hq // Hkv)], v[b][j, h // (Hq // Hkv)]
                s = kk @ q[b, i, h] * scale
                m = s.max()
                p = np.exp(s - m)
                lse[b, i, h] = m + np.log(p.sum())
                p /= p.sum()
                o[b, i, h] = p @ vv
                mass[b, i, h] = p @ np.abs(vv)
                qk[b, i, h] = (np.abs(kk) @ np.abs(q[b, i, h])).max() * scale
    return o, lse, mass, qk


def attention_bounds(dtype, n, o, lse, mass, qk, d, vmax):
    """How far o and lse may be off.  A score is a sum of d products: off by (d + 4)
    2^-24 sum |q k| with its scale and its logarithm's base; a weight by that, the
    subtraction of the maximum (its size at most twice qk) and the hardware's exp2 (2^-22);
    a sum of n by n 2^-24 of its terms' sizes, the pieces' factors (exp2 each) by 2^-20
    altogether.  bf16: each weight half a step more, O half a step.  A weight below 2^-126 of
    the largest is no normal fp32 number and may be lost whole: n of them times the largest
    value, vmax (where every heavier token's V is 0, they are all there is of O)."""
    w = qk * (d + 4 + 4 + 4) * 2.0 ** -24 + 2.0 ** -22 + 2.0 ** -20
    rel = 2 * w + (2 * n + 16) * 2.0 ** -24
    ob = mass * rel[..., None] + np.abs(o) * HALF["f32"] + n * vmax * 2.0 ** -126
    if dtype == "bf16":
        ob = ob + (mass + np.abs(o)) * HALF["bf16"] * (1 + 2.0 ** -7)
    lb = w + (n + 16) * 2.0 ** -24 + np.abs(np.where(np.isfinite(lse), lse, 0)) * 2.0 ** -22
    return ob, lb


def prob(x):
    x = np.asarray(x, np.float64)
    return np.where(np.isfinite(x) & (x > 0), x, 0.0)


def spec_accept(p, q, draft, u):
    """p [B, L, V], q [B, L - 1, V] or None, as float64 of the stored values."""
    B, L, V = p.shape
    p = prob(p)
    q = None if q is None else prob(q)
    kept, tokens = np.zeros(B, np.int64), np.full((B, L), -1, np.int64)
    for b in range(B):
        a = 0
        while a < L - 1:
            t = int(draft[b, a])
            if not (0 <= t < V) or not u[b, a] * (1.0 if q is None else q[b, a, t]) < p[b, a, t]:
                break
            a += 1
        r = p[b, a].copy()
        if a < L - 1:
            if q is not None:
                r -= q[b, a]
            elif 0 <= draft[b, a] < V:
                r[draft[b, a]] -= 1.0
            r = np.maximum(r, 0.0)
        if not r.any():
            r = p[b, a]
        some = np.flatnonzero(r)
        cdf = np.cumsum(r)
        past = np.flatnonzero((cdf > u[b, L - 1] * cdf[-1]) & (r > 0))
        kept[b] = a
        tokens[b, :a] = draft[b, :a]
        tokens[b, a] = past[0] if len(past) else (some[-1] if len(some) else 0)
    return kept, tokens


def norm_rope(x, w, pos, inv, norm=True, eps=1e-6, interleaved=False):
    """x [B, n, H, d], pos [B, n].  Returns the rows, and |y1| + |y2| for error bounds."""
    x = x.astype(np.float64)
    if norm:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
        if w is not None:
            x = x * w
    r = 2 * len(inv)
    t = (pos[..., None].astype(np.float64) * inv.astype(np.float64))[:, :, None]
    y, size = x.copy(), np.abs(x)
    one, two = ((slice(0, r, 2), slice(1, r, 2)) if interleaved
                else (slice(0, r // 2), slice(r // 2, r)))
    y1, y2 = x[..., one], x[..., two]
    y[..., one] = y1 * np.cos(t) - y2 * np.sin(t)
    y[..., two] = y2 * np.cos(t) + y1 * np.sin(t)
    size[..., one] = size[..., two] = np.abs(y1) + np.abs(y2)
    return y, size


def norm_rope_bound(dtype, y, size, d):
    """The sum of d squares is off by d 2^-24 at most, half of it after the root; root,
    quotient, two products, the angle's rounding (pi 2^-24), sine and cosine (2 ulp), two
    products and a sum: 16 more.  Then the result's rounding."""
    return size * (d / 2 + 16) * 2.0 ** -24 + np.abs(y) * HALF[dtype] * (1 + 2.0 ** -7)
