"""Norm of query and key heads with the rotation, on the GPU, against float64 with error
bounds from the arithmetic (plain_ops.py)."""
import numpy as np
import pytest
import torch

import paper_2408_11049_amd as md
import plain_ops as plain

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def host(t):
    return None if t is None else t.detach().to(torch.float64).cpu().numpy()


def randn(shape, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(shape, generator=g).to(DT[dtype]).to(DEV)


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def inv_freq(rot, base=10000.0):
    return (base ** (-torch.arange(0, rot, 2, dtype=torch.float64) / max(rot, 1))).float().to(DEV)


def same(got, x, w, pos, inv, dtype, **kw):
    y, size = plain.norm_rope(host(x), host(w), pos, inv.double().cpu().numpy(), **kw)
    err, tol = np.abs(host(got) - y), plain.norm_rope_bound(dtype, y, size, x.shape[3])
    assert (err <= tol).all(), f"{np.max(err / np.maximum(tol, 1e-300)):.2f} times the bound off"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("B,n,Hq,Hkv,share", [(1, 1, 1, 1, 1.0), (2, 5, 8, 2, 0.5), (3, 7, 7, 1, 1.0),
                                              (1, 300, 33, 3, 0.25), (300, 1, 4, 4, 0.0)])
def test_rows(dtype, d, interleaved, B, n, Hq, Hkv, share):
    q, k = randn((B, n, Hq, d), dtype, 1), randn((B, n, Hkv, d), dtype, 2)
    qw, kw = randn((d,), dtype, 3), randn((d,), dtype, 4)
    inv = inv_freq(int(d * share))
    pos0 = np.random.default_rng(n).integers(0, 5000, B)
    pos = pos0[:, None] + np.arange(n)
    qo, ko, lens = md.md_qk_norm_rope(q, k, ints(pos0.tolist()), inv, q_weight=qw, k_weight=kw,
                                      interleaved=interleaved)
    same(qo, q, qw, pos, inv, dtype, interleaved=interleaved)
    same(ko, k, kw, pos, inv, dtype, interleaved=interleaved)
    assert lens.tolist() == (pos0 + n).tolist()


@pytest.mark.parametrize("norm,weights,eps", [(False, False, 0.0), (True, False, 1e-5),
                                              (True, True, 0.0), (True, True, 10.0)])
def test_norms(norm, weights, eps):
    q, k = randn((2, 3, 4, 128), "f32", 5), randn((2, 3, 2, 128), "f32", 6)
    q[0, 0, 0] = 0                    # a row of zeros stays zero where eps is not
    q[1, 1] *= 1e-4
    q[1, 2] *= 1e6
    w = randn((128,), "f32", 7) if weights else None
    if eps == 0.0:
        q[0, 0, 0, 3] = 1.0
    inv, pos = inv_freq(128), np.array([[0, 1, 2], [9, 10, 11]])
    qo, ko, _ = md.md_qk_norm_rope(q, k, ints([0, 9]), inv, norm=norm, q_weight=w, k_weight=w,
                                   eps=eps)
    same(qo, q, w, pos, inv, "f32", norm=norm, eps=eps)
    same(ko, k, w, pos, inv, "f32", norm=norm, eps=eps)


@pytest.mark.parametrize("start", [-3, 0, 131072, 10 ** 7 + 1, 2 ** 31 - 40])
def test_far_positions(start):
    """The angle's fraction of a turn is kept at any position (32 bits would lose it)."""
    q, k = randn((1, 9, 2, 64), "f32", 8), randn((1, 9, 1, 64), "f32", 9)
    inv = inv_freq(64, 500000.0)
    qo, ko, _ = md.md_qk_norm_rope(q, k, ints([start]), inv, norm=False)
    pos = start + np.arange(9, dtype=np.int64)[None]
    same(qo, q, None, pos, inv, "f32", norm=False)
    same(ko, k, None, pos, inv, "f32", norm=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [0, 1, 16])
def test_into_the_cache(dtype, page):
    """Fused with the append: the same cache as norm and rotation, then md_kv_append, bit for
    bit; rows outside the cache are left out; q, k and v are views of one projection."""
    B, n, Hq, Hkv, d, cap = 4, 5, 6, 2, 128, 32
    qkv = randn((B, n, (Hq + 2 * Hkv) * d), dtype, 1)
    q, k, v = (x.unflatten(2, (-1, d)) for x in qkv.split([Hq * d, Hkv * d, Hkv * d], 2))
    qw, kw, inv = randn((d,), dtype, 2), randn((d,), dtype, 3), inv_freq(d)
    pos0 = ints([0, 27, 30, -2])
    pt = None
    shape = (B, cap, Hkv, d)
    if page:
        shape = (B * cap // page + 2, page, Hkv, d)
        pt = torch.randperm(B * cap // page).to(torch.int32).view(B, -1).to(DEV)
        pt[0, 3 // page] = 10 ** 6
    caches = [randn(shape, dtype, 4 + i) for i in range(2)]
    ck, cv = [t.clone() for t in caches]
    want_q, rows, _ = md.md_qk_norm_rope(q, k, pos0, inv, q_weight=qw, k_weight=kw)
    md.md_kv_append(*caches, rows, v.contiguous(), pos0, page_table=pt)
    k_out = torch.empty_like(rows)
    qo, ko, lens = md.md_qk_norm_rope(q, k, pos0, inv, q_weight=qw, k_weight=kw, v_new=v, k=ck, v=cv,
                                      page_table=pt, k_out=k_out)
    assert ko is k_out and torch.equal(ko, rows) and torch.equal(qo, want_q)
    assert torch.equal(ck, caches[0]) and torch.equal(cv, caches[1])
    assert lens.tolist() == [5, 32, 35, 3]
    same(qo, q, qw, pos0.cpu().numpy()[:, None] + np.arange(n), inv, dtype)
    _, none, _ = md.md_qk_norm_rope(q, k, pos0, inv, q_weight=qw, k_weight=kw, v_new=v, k=ck, v=cv,
                                    page_table=pt)
    assert none is None and torch.equal(ck, caches[0])


def test_in_place():
    q, k, pos0, inv = randn((3, 4, 9, 64), "bf16", 1), randn((3, 4, 2, 64), "bf16", 2), ints([1, 2, 3]), inv_freq(32)
    qo, ko, _ = md.md_qk_norm_rope(q, k, pos0, inv)
    md.md_qk_norm_rope(q, k, pos0, inv, q_out=q, k_out=k)
    assert torch.equal(q, qo) and torch.equal(k, ko)


def test_value_rows_move_bit_for_bit():
    v = torch.full((1, 2, 1, 64), float("nan"), dtype=torch.bfloat16, device=DEV)
    v.view(torch.int16)[0, 1] = torch.arange(64, dtype=torch.int16, device=DEV) - 0x7fc0 % 64 + 0x7f80
    q = randn((1, 2, 1, 64), "bf16", 1)
    ck, cv = (torch.zeros((1, 4, 1, 64), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    md.md_qk_norm_rope(q, q.clone(), ints([1]), inv_freq(64), v_new=v, k=ck, v=cv)
    assert torch.equal(cv.view(torch.int16)[0, 1:3], v.view(torch.int16)[0])
    assert not cv[0, 0].any() and not cv[0, 3].any() and not ck[0, 3].any()


def test_nan_stays_in_its_row():
    q, k = randn((1, 2, 3, 64), "f32", 1), randn((1, 2, 2, 64), "f32", 2)
    q[0, 1, 2, 5] = float("nan")
    k[0, 0, 1, 63] = float("inf")
    qo, ko, _ = md.md_qk_norm_rope(q, k, ints([3]), inv_freq(64))
    bad = torch.zeros((1, 2, 3), dtype=torch.bool, device=DEV)
    bad[0, 1, 2] = True
    assert torch.equal(torch.isnan(qo).any(-1), bad)
    assert torch.isnan(ko[0, 0, 1]).any() and torch.isfinite(ko[0, 1]).all()


def test_streams_and_graph():
    q, k, v = (randn((2, 3, h, 128), "bf16", h) for h in (8, 2, 3))
    v = v[:, :, :2].contiguous()
    pos0, inv = ints([0, 7]), inv_freq(128)
    ck, cv = (torch.zeros((2, 64, 2, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    q_out, lens = torch.empty_like(q), torch.empty_like(pos0)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    a = [md.md_qk_norm_rope(q, k, pos0, inv, stream=s) for _ in range(3)]
    torch.cuda.synchronize()
    b = md.md_qk_norm_rope(q, k, pos0, inv)
    assert all(torch.equal(x[0], b[0]) and torch.equal(x[1], b[1]) for x in a)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        md.md_qk_norm_rope(q, k, pos0, inv, v_new=v, k=ck, v=cv, q_out=q_out, lens_out=lens)
    for seed, at in ((1, [0, 7]), (2, [3, 50]), (3, [61, 0])):
        q.copy_(randn(q.shape, "bf16", 20 + seed))
        pos0.copy_(ints(at))
        g.replay()
        torch.cuda.synchronize()
        wk, wv = torch.zeros_like(ck), torch.zeros_like(cv)
        want, _, wl = md.md_qk_norm_rope(q, k, pos0, inv, v_new=v, k=wk, v=wv)
        assert torch.equal(q_out, want) and torch.equal(lens, wl)
        for x, y in ((ck, wk), (cv, wv)):
            for i, p in enumerate(at):
                assert torch.equal(x[i, p:p + 3], y[i, p:p + 3])


def test_binding_refusals():
    q, k, pos0, inv = randn((2, 2, 4, 64), "bf16", 1), randn((2, 2, 2, 64), "bf16", 2), ints([0, 0]), inv_freq(64)
    c = torch.zeros((2, 8, 2, 64), dtype=torch.bfloat16, device=DEV)
    f = md.md_qk_norm_rope
    w = torch.ones(64, dtype=torch.bfloat16, device=DEV)
    buf = torch.empty(q.numel() + 64, dtype=q.dtype, device=DEV)
    for i, bad in enumerate([
            lambda: f(q.cpu(), k, pos0, inv), lambda: f(q, k.cpu(), pos0, inv),
            lambda: f(q, k.float(), pos0, inv), lambda: f(q.half(), k.half(), pos0, inv),
            lambda: f(q, k, pos0.long(), inv), lambda: f(q, k, pos0, inv.double()),
            lambda: f(q, k, pos0, inv[:3]), lambda: f(q, k, pos0, inv_freq(128)),
            lambda: f(q, k, pos0, inv, eps=-1.0), lambda: f(q, k, pos0, inv, eps=float("nan")),
            lambda: f(q, k, pos0, inv, q_weight=w.float()), lambda: f(q, k, pos0, inv, k_weight=w[:32]),
            lambda: f(q, k, pos0, inv, norm=False, q_weight=w),
            lambda: f(q, k, pos0, inv, v_new=k), lambda: f(q, k, pos0, inv, k=c, v=c.clone()),
            lambda: f(q, k, pos0, inv, v_new=k, k=c.float(), v=c.float()),
            lambda: f(q, k, pos0, inv, v_new=k, k=c[:, :, :1], v=c[:, :, :1]),
            lambda: f(q, k, pos0, inv, page_table=ints([[0], [1]])),
            lambda: f(q[..., :48], k[..., :48], pos0, inv_freq(48)),
            lambda: f(q.transpose(2, 3), k, pos0, inv),
            lambda: f(q, k, pos0, inv, lens_out=pos0),
            lambda: f(buf[: q.numel()].view(q.shape), k, pos0, inv, q_out=buf[64:].view(q.shape)),
            lambda: f(q, k, pos0, inv, q_out=torch.empty_like(k)),
            lambda: f(q, k, pos0, inv, k_out=k.view(2, 2, 1, 128))]):
        with pytest.raises(ValueError):
            bad()
            pytest.fail(f"case {i} was accepted")


def test_no_new_token_still_gives_the_lengths():
    q, k = randn((3, 0, 4, 64), "bf16", 0), randn((3, 0, 2, 64), "bf16", 1)
    a, b, lens = md.md_qk_norm_rope(q, k, ints([4, 0, 9]), inv_freq(64))
    assert a.shape == q.shape and b.shape == k.shape and lens.tolist() == [4, 0, 9]


def test_more_tokens_than_one_grid_dimension_counts():
    """Rows of the ends and of the middle against the same rows in a small call."""
    n = (1 << 23) + 77
    q = torch.randn((1, n, 1, 64), dtype=torch.bfloat16, device=DEV)
    k = torch.randn((1, n, 1, 64), dtype=torch.bfloat16, device=DEV)
    a, b, lens = md.md_qk_norm_rope(q, k, ints([3]), inv_freq(64))
    assert lens.tolist() == [n + 3]
    for at in (0, (1 << 22) - 40, (1 << 23) - 60, n - 70):
        s = slice(at, at + 70)
        ra, rb, _ = md.md_qk_norm_rope(q[:, s], k[:, s], ints([3 + at]), inv_freq(64))
        assert torch.equal(a[:, s], ra) and torch.equal(b[:, s], rb)
