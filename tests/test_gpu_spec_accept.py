"""Sampled acceptance on the GPU against a float64 reference: whole numbers, equal."""
import numpy as np
import pytest
import torch

import paper_2408_11049_amd as md
import plain_ops as plain

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def host(t):
    return None if t is None else t.to(torch.float64).cpu().numpy()


def make(B, g, V, dtype, seed, sampled=True):
    rng = np.random.default_rng(seed)
    t = rng.standard_normal((B, g + 1, V)) * 2

    def softmax(x):
        x = np.exp(x - x.max(-1, keepdims=True))
        return torch.from_numpy(x / x.sum(-1, keepdims=True)).to(DT[dtype]).to(DEV)

    p = softmax(t)
    q = softmax(t[:, :g] + 0.5 * rng.standard_normal((B, g, V))) if sampled else None
    draft = rng.integers(0, V, (B, g))
    top = t[:, :g].argmax(-1)
    draft = np.where(rng.random((B, g)) < 0.8, top, draft).astype(np.int32)
    u = rng.random((B, g + 1)).astype(np.float32)
    return p, q, torch.from_numpy(draft).to(DEV), torch.from_numpy(u).to(DEV)


def check(p, q, draft, u, **kw):
    B, L = u.shape
    acc = torch.full((B,), -99, dtype=torch.int32, device=DEV)
    tok = torch.full((B, L), -99, dtype=torch.int32, device=DEV)
    md.md_spec_accept(p, q, draft, u, accepted=acc, tokens=tok, **kw)
    a, t = plain.spec_accept(host(p), host(q), draft.cpu().numpy(), host(u))
    assert acc.tolist() == a.tolist()
    assert tok.tolist() == t.tolist()
    return acc, tok


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("sampled", [True, False])
@pytest.mark.parametrize("B,g,V", [(1, 1, 1), (3, 4, 2), (5, 0, 17), (2, 3, 2049), (17, 5, 4096),
                                   (4, 8, 32003), (1, 4, 128256), (2, 70, 100), (9, 2, 16392)])
def test_shapes(dtype, sampled, B, g, V):
    for seed in range(3):
        check(*make(B, g, V, dtype, seed, sampled))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("sampled", [True, False])
@pytest.mark.parametrize("B,V", [(3, 50257), (2, 65535), (2, 65537), (3, 70001), (1, (1 << 20) + 4099)])
def test_rows_that_end_inside_a_vector(dtype, sampled, B, V):
    """Rows that start and end anywhere, in one launch and in two; draws from the last tokens and
    from all over."""
    for last in (None, 1 - 2.0 ** -24, 1 - 2.0 ** -17, 0.0):
        p, q, draft, u = make(B, 2, V, dtype, V % 7, sampled)
        if last is not None:
            u[:, -1] = last
        check(p, q, draft, u)
        heavy = p.clone()  # the mass on the row's last tokens
        heavy[:, :, -3:] = 0.25
        check(heavy, q, draft, u)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_draws_at_the_borders(dtype):
    """Probabilities that are powers of two, sums and products exact: u on every border."""
    V, g = 16, 1
    p = torch.full((17, 2, V), 1 / 16, dtype=DT[dtype], device=DEV)
    q = torch.zeros((17, 1, V), dtype=DT[dtype], device=DEV)
    q[:, 0, :8] = 1 / 8
    draft = torch.full((17, 1), 3, dtype=torch.int32, device=DEV)
    u = torch.zeros((17, 2), device=DEV)
    u[:, 0] = 0.5                       # u q = p exactly: not below, refused
    u[:, 1] = torch.arange(17) / 16     # r = 1/16 on 8..15; the last u is 1
    acc, tok = check(p, q, draft, u)
    assert acc.tolist() == [0] * 17
    assert tok[:, 0].tolist() == [8 + k // 2 for k in range(16)] + [15]
    u[:, 0] = 0.5 - 2.0 ** -20          # just below: kept, the bonus from p's own row
    acc, tok = check(p, q, draft, u)
    assert acc.tolist() == [1] * 17 and tok[:, 1].tolist() == list(range(16)) + [15]


def test_rows_with_nothing_left():
    """p = q (no residual): p itself; p all 0: token 0; q = 0 at the draft; p = 0 there."""
    V = 300
    p = torch.zeros((5, 2, V), device=DEV)
    q = torch.zeros((5, 1, V), device=DEV)
    p[0, 0, 7] = q[0, 0, 7] = 1.0       # draft elsewhere: refused, r = 0, p's row: 7
    p[2, 0, 5], q[2, 0, 9] = 0.25, 1.0  # q(d) = 0, p(d) > 0: kept
    p[3, 0, 4], q[3, 0, 6] = 1.0, 1.0   # p(d) = 0: refused, r on 4
    p[2, 1, 299] = 0.5
    draft = torch.tensor([[8], [0], [5], [6], [2]], dtype=torch.int32, device=DEV)
    u = torch.full((5, 2), 0.75, device=DEV)
    acc, tok = check(p, q, draft, u)
    assert acc.tolist() == [0, 0, 1, 0, 0]
    assert tok.tolist() == [[7, -1], [0, -1], [5, 299], [4, -1], [0, -1]]


def test_values_that_are_no_probabilities():
    """NaN, infinities and negatives count as 0; drafts outside the vocabulary (padding) are
    refused, with rows of zeros for them the target's own row is drawn from."""
    p, q, draft, u = make(6, 3, 1000, "f32", 5)
    p[0, 0, 3], p[0, 0, 5], p[1, 0, 7] = float("nan"), float("inf"), -4.0
    q[0, 0, 9], q[1, 0, 11], q[2, 0, 13] = float("nan"), float("inf"), -1.0
    draft[0, 0], draft[1, 0], draft[2, 0] = 3, 11, 13
    draft[3, 1], draft[4, 0], draft[5, 2] = -1, 1000, 2 ** 31 - 1
    q[3, 1:] = 0
    q[4] = 0
    check(p, q, draft, u)
    check(p, None, draft, u)
    u[0], u[1], u[2] = float("nan"), -1.0, 2.0
    got, _ = md.md_spec_accept(p, q, draft, u)
    assert got[0] == 0


def test_sums_of_many_small_terms():
    """A flat row of 10^5 tokens: 32-bit sums would misplace most of the draws."""
    V, B = 100003, 64
    p = torch.rand((B, 1, V), device=DEV, generator=torch.Generator(DEV).manual_seed(1)) / V
    u = torch.rand((B, 1), device=DEV, generator=torch.Generator(DEV).manual_seed(2))
    check(p, None, torch.empty((B, 0), dtype=torch.int32, device=DEV), u)


def test_millions_of_sequences():
    B = (1 << 22) - 1
    p = torch.ones((B, 1, 2), device=DEV)
    u = torch.zeros((B, 1), device=DEV)
    u[1::2] = 0.75
    acc, tok = md.md_spec_accept(p, None, torch.empty((B, 0), dtype=torch.int32, device=DEV), u)
    assert int(acc.abs().sum()) == 0
    assert torch.equal(tok[:, 0], (torch.arange(B, device=DEV) % 2).to(torch.int32))


def test_unaligned_rows_and_given_buffers():
    p, q, draft, u = make(3, 2, 4096, "bf16", 9)
    flat = torch.empty(p.numel() + 1, dtype=p.dtype, device=DEV)
    flat[1:] = p.flatten()
    ws = torch.full((1 << 16,), 255, dtype=torch.uint8, device=DEV)
    check(flat[1:].view(p.shape), q, draft, u, workspace=ws)


def test_distribution_is_the_targets():
    """Over many draws the first token follows p, whatever q: Pearson's statistic of 16
    cells over 2^16 draws is below 60 (15 degrees of freedom: 2e-7)."""
    V, B = 16, 1 << 16
    rng = np.random.default_rng(3)
    p = rng.random(V) ** 2
    q = rng.random(V) ** 2
    p, q = p / p.sum(), q / q.sum()
    P = torch.tensor(p, dtype=torch.float32, device=DEV).expand(B, 2, V).contiguous()
    Q = torch.tensor(q, dtype=torch.float32, device=DEV).expand(B, 1, V).contiguous()
    draft = torch.from_numpy(rng.choice(V, (B, 1), p=q).astype(np.int32)).to(DEV)
    u = torch.from_numpy(rng.random((B, 2)).astype(np.float32)).to(DEV)
    _, tok = md.md_spec_accept(P, Q, draft, u)
    seen = np.bincount(tok[:, 0].cpu().numpy(), minlength=V)
    assert ((seen - B * p) ** 2 / (B * p)).sum() < 60


def test_streams_and_graph():
    p, q, draft, u = make(8, 4, 5000, "f32", 11)
    acc, tok = torch.empty(8, dtype=torch.int32, device=DEV), torch.empty((8, 5), dtype=torch.int32, device=DEV)
    ws = torch.empty(1 << 16, dtype=torch.uint8, device=DEV)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = [md.md_spec_accept(p, q, draft, u, stream=s) for _ in range(4)]
    torch.cuda.synchronize()
    want = md.md_spec_accept(p, q, draft, u)
    assert all(torch.equal(a, want[0]) and torch.equal(t, want[1]) for a, t in got)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        md.md_spec_accept(p, q, draft, u, accepted=acc, tokens=tok, workspace=ws)
    for seed in (1, 2, 3):
        for x, y in zip((p, q, draft, u), make(8, 4, 5000, "f32", seed)):
            x.copy_(y)
        g.replay()
        torch.cuda.synchronize()
        a, t = plain.spec_accept(host(p), host(q), draft.cpu().numpy(), host(u))
        assert acc.tolist() == a.tolist() and tok.tolist() == t.tolist()


def test_binding_refusals():
    p, q, draft, u = make(2, 2, 64, "f32", 1)
    f = md.md_spec_accept
    for i, bad in enumerate([
            lambda: f(p.cpu(), q, draft, u), lambda: f(p, q.cpu(), draft, u),
            lambda: f(p, q.bfloat16(), draft, u), lambda: f(p.half(), None, draft, u),
            lambda: f(p, q, draft.long(), u), lambda: f(p, q, draft, u.double()),
            lambda: f(p, q, draft, u[:, :2]), lambda: f(p, q[:, :1], draft, u),
            lambda: f(p.transpose(0, 1), q, draft, u),
            lambda: f(p, q, draft, u, accepted=torch.empty(1, dtype=torch.int32, device=DEV)),
            lambda: f(p, q, draft, u, tokens=torch.empty(5, dtype=torch.int32, device=DEV)),
            lambda: f(p, q, draft, u, workspace=torch.empty(1 << 20, dtype=torch.uint8)),
            lambda: f(torch.ones((1, 1, 100000), device=DEV), None, draft[:1, :0], u[:1, :1],
                      workspace=torch.empty(64, dtype=torch.uint8, device=DEV))]):
        with pytest.raises(ValueError):
            bad()
            pytest.fail(f"case {i} was accepted")
