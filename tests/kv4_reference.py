"""Attention over a 4-bit cache in float64 torch, for contexts that loops over numpy rows would
take too long for: elementary products and sums, no code of the library."""
import torch

import plain_ops as plain


def rows(codes, scales, pt, b):
    """Sequence b's values in token order, [S, Hkv, d] float64."""
    if pt is None:
        c, s = codes[b], scales[b]
    else:
        ids = pt[b].long()
        c, s = codes[ids].flatten(0, 1), scales[ids].flatten(0, 1)
    level = torch.tensor(list(plain.LEVELS) + list(-plain.LEVELS), dtype=torch.float64,
                         device=codes.device)
    v = level[torch.stack([c & 15, c >> 4], -1).flatten(-2).long()]
    return v * torch.exp2(s.double() - 127).repeat_interleave(32, -1)


def attention(q, cache, pt, lens, n_sink=0, window=None, scale=None):
    """q [B, L, Hq, d], cache (k, v, k_scale, v_scale) without NaN or infinite values.  Returns
    what plain.attention does, as numpy float64, and the largest |V| of any sequence."""
    B, L, Hq, d = q.shape
    Hkv = cache[0].shape[2]
    G = Hq // Hkv
    dev = q.device
    scale = scale or d ** -0.5
    o = torch.zeros((B, L, Hq, d), dtype=torch.float64, device=dev)
    mass, qk = torch.zeros_like(o), torch.zeros((B, L, Hq), dtype=torch.float64, device=dev)
    lse = torch.full_like(qk, -float("inf"))
    vmax = 0.0
    for b, S in enumerate(lens):
        if S <= 0:
            continue
        k, v = rows(cache[0], cache[2], pt, b)[:S], rows(cache[1], cache[3], pt, b)[:S]
        vmax = max(vmax, float(v.abs().max()))
        pos = (torch.arange(L, device=dev) + S - L)[:, None]
        j = torch.arange(S, device=dev)[None]
        see = j <= pos
        if window is not None:
            see = see & ((j < n_sink) | (j > pos - window))
        see = see.repeat_interleave(G, 0)  # row i * G + g
        some = see.any(1)
        for h in range(Hkv):
            qh = q[b, :, h * G:(h + 1) * G].reshape(L * G, d).double()
            kh, vh = k[:, h].contiguous(), v[:, h].contiguous()
            s = (qh @ kh.t()) * scale
            s = torch.where(see, s, -float("inf"))
            m = torch.where(some, s.max(1).values, 0.0)
            p = torch.exp(s - m[:, None])
            total = p.sum(1)
            p = p / torch.where(some, total, 1.0)[:, None]
            at = (b, slice(None), slice(h * G, (h + 1) * G))
            o[at] = (p @ vh).view(L, G, d)
            mass[at] = (p @ vh.abs()).view(L, G, d)
            lse[at] = torch.where(some, m + total.log(), -float("inf")).view(L, G)
            size = torch.where(see, (qh.abs() @ kh.abs().t()) * scale, 0.0)
            qk[at] = size.max(1).values.view(L, G)
    return *(t.cpu().numpy() for t in (o, lse, mass, qk)), vmax
