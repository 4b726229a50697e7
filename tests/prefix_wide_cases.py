"""Calls of md_prefix_attn whose groups of many rows share short prefixes in the tiles that the waves of a workgroup
share, and their float64 oracle.  Tiles hold 64 keys, in blocks of 32.

Each row looks for one key (its weight there is most of the row's: the keys at tile ends, part ends and the
last ones, in turn), or away from all of them (each of its scores is near -8, so that a key that is none, of score 0,
would outweigh the rest)."""
import numpy as np
import torch

import plain_answers as plain

# name: Hq, Hkv, d, L, sequences a prefix, own page, prefix page, bound on the prefixes, their lengths;
# the parts of a prefix that the plan has to make at 256 compute units.
ONE_PART = [520, 519, 513, 512, 511, 449, 448, 447, 385, 384, 321, 320, 319, 257, 256, 255, 200, 193, 192, 191, 130, 129,
            128, 127, 97, 96, 65, 64, 63, 33, 1, 0]
CASES = {
    "one part, 168 rows": ((64, 8, 128, 3, 7, 0, 0, 520, ONE_PART), 1),
    "one part, 168 rows, pages of 4": ((64, 8, 128, 3, 7, 16, 4, 520, ONE_PART), 1),
    "one part, 240 rows, 64 channels, pages of 8": ((32, 8, 64, 4, 15, 16, 8, 520, ONE_PART), 1),
    "eight parts, 200 rows": ((32, 8, 128, 2, 25, 16, 16, 4096, [4096, 517, 2049, 4033]), 8),
    "eight parts, 200 rows, 64 channels": ((32, 8, 64, 2, 25, 0, 0, 4096, [1087, 4095, 577, 576]), 8),
    "four parts, 960 rows": ((64, 8, 128, 8, 15, 0, 16, 2048, [2047, 130]), 4),
    "two parts, 264 rows": ((32, 8, 128, 2, 33, 0, 0, 1024, [1024, 993, 961, 959, 97, 33, 32, 0]), 2),
    "two parts, 384 rows, 64 channels": ((32, 8, 64, 4, 24, 16, 16, 1024, [1023, 992, 129, 96, 65, 64, 31, 1]), 2),
    "sixteen parts, 288 rows": ((32, 8, 128, 4, 18, 16, 16, 8192, [700]), 16),
    "sixteen parts, 288 rows, 64 channels": ((32, 8, 64, 4, 18, 0, 0, 8192, [2015]), 16),
}


def edges(T, parts):
    """Keys at which tiles, blocks and parts of a prefix of T tokens begin and end."""
    tiles = -(-T // 64)
    at = [tiles * c // parts * 64 for c in range(1, parts)]
    at += [32, 64, 128, T // 64 * 64, T // 32 * 32, T // 64 * 64 - 64, T]
    keys = [0, T - 1, T - 2] + [x for a in at for x in (a - 1, a)]
    return list(dict.fromkeys(x for x in keys if 0 <= x < T))


class Inputs:
    """Host tensors: q [B, L, Hq, d], and the rows of own caches and prefixes, bf16, as lists of [S, Hkv, d]."""

    def __init__(self, name):
        (self.Hq, self.Hkv, self.d, self.L, self.n, self.page, self.ppage, self.bound, self.plens), self.parts = CASES[name]
        gen = torch.Generator().manual_seed(len(name))
        self.B, G = self.n * len(self.plens), self.Hq // self.Hkv
        self.lens = [self.L + b % 9 for b in range(self.B)]

        def rows(lens, mean):
            return [(torch.randn((s, self.Hkv, self.d), generator=gen) + mean).to(torch.bfloat16) for s in lens]
        self.k, self.v, self.pk, self.pv = rows(self.lens, 0.7), rows(self.lens, 0.0), rows(self.plens, 0.7), rows(self.plens, 0.0)
        self.q = torch.full((self.B, self.L, self.Hq, self.d), -(8.0 / 0.7) * self.d ** -0.5)
        for b in range(self.B):
            T = self.plens[b // self.n]
            at = edges(T, self.parts)
            for i in range(self.L):
                for h in range(self.Hq):
                    r = ((b % self.n) * self.L + i) * G + h % G
                    if at and r % 5:
                        key = self.pk[b // self.n][at[(r - r // 5) % len(at)], h // G].float()
                        self.q[b, i, h] = (key - 0.7) * (12.0 * self.d ** -0.5)
        self.q = self.q.to(torch.bfloat16)

    def oracle(self, p, k=None, v=None):
        """o, lse and their bounds for the sequences of prefix p, whose rows may be given."""
        k, v = (self.pk[p] if k is None else k), (self.pv[p] if v is None else v)
        k, v = k.double(), v.double()
        n, L, G, d = self.n, self.L, self.Hq // self.Hkv, self.d
        shape = (n, L, self.Hq)
        o, lse, mass, qk = np.zeros(shape + (d,)), np.zeros(shape), np.zeros(shape + (d,)), np.zeros(shape)
        for x in range(n):
            b = p * n + x
            S = self.lens[b]
            for h in range(self.Hkv):
                kk = torch.cat([k[:, h], self.k[b][:, h].double()])
                vv = torch.cat([v[:, h], self.v[b][:, h].double()])
                q = self.q[b, :, h * G:(h + 1) * G].double().reshape(L * G, d)
                s = q @ kk.T.contiguous() * d ** -0.5
                last = len(k) + S - L + torch.arange(L).repeat_interleave(G)
                s[torch.arange(len(kk))[None] > last[:, None]] = -np.inf
                z = torch.logsumexp(s, 1)
                w = torch.exp(s - z[:, None])
                heads = slice(h * G, (h + 1) * G)
                o[x, :, heads] = (w @ vv).reshape(L, G, d).numpy()
                mass[x, :, heads] = (w @ vv.abs()).reshape(L, G, d).numpy()
                lse[x, :, heads] = z.reshape(L, G).numpy()
                qk[x, :, heads] = ((q.abs() @ kk.abs().T.contiguous()).amax(1) * d ** -0.5).reshape(L, G).numpy()
        top = float(max(v.abs().max() if len(v) else 0, max(r.abs().max() for r in self.v)))
        return (o, lse) + plain.prefix_bounds("bf16", len(k) + max(self.lens), o, lse, mass, qk, d, top)
