"""The torch reference of the 4-bit attention against the numpy one, on the CPU."""
import numpy as np
import pytest
import torch

import kv4_reference
import plain_ops as plain


@pytest.mark.parametrize("page", [0, 8])
@pytest.mark.parametrize("n_sink,window", [(0, None), (3, 20), (0, 1)])
def test_two_references_agree(page, n_sink, window):
    rng = np.random.default_rng(page)
    B, L, Hq, Hkv, d, S = 4, 5, 6, 2, 64, 48
    blocks, toks = (B * S // page, page) if page else (B, S)
    cache = [torch.from_numpy(rng.integers(0, 256, (blocks, toks, Hkv, w)).astype(np.uint8))
             for w in (d // 2, d // 2)]
    cache += [torch.from_numpy(rng.integers(124, 128, (blocks, toks, Hkv, d // 32)).astype(np.uint8))
              for _ in range(2)]
    pt = torch.from_numpy(rng.permutation(blocks).reshape(B, -1)) if page else None
    q = torch.from_numpy(rng.standard_normal((B, L, Hq, d)))
    lens = [48, 3, 0, 17]
    got = kv4_reference.attention(q, cache, pt, lens, n_sink, window, 0.3)
    kv = []
    for c, s in ((cache[0], cache[2]), (cache[1], cache[3])):
        x = plain.kv4_values(plain.unpack(c.numpy()), s.numpy().astype(np.int64))
        if page:
            x = x[pt.numpy()].reshape(B, S, Hkv, d)
        kv.append(list(x))
    want = plain.attention(q.numpy(), *kv, lens, n_sink, window, 0.3)
    for a, b in zip(got, want):
        assert np.array_equal(np.isfinite(a), np.isfinite(b))
        fin = np.isfinite(b)
        assert np.allclose(a[fin], b[fin], rtol=1e-12, atol=1e-12)
    assert got[4] == max(np.abs(v[:n]).max() for v, n in zip(kv[1], lens) if n)
