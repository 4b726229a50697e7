"""Sampled acceptance of rows over 65536 tokens on the GPU: the segments' sums pass from one
launch to the next through the workspace, in workspaces of any contents, on streams and in
graphs."""
import numpy as np
import pytest
import torch

import paper_2408_11049_amd as md
import plain_ops as plain
from test_gpu_spec_accept import DEV, check, host, make

pytestmark = pytest.mark.gpu


def need(B, g, V):
    n = md.load_library().md_spec_accept_workspace_bytes(B, g, V)
    assert n > 0
    return n


def outputs(B, g):
    return (torch.empty(B, dtype=torch.int32, device=DEV),
            torch.empty((B, g + 1), dtype=torch.int32, device=DEV))


def reference(p, q, draft, u):
    a, t = plain.spec_accept(host(p), host(q), draft.cpu().numpy(), host(u))
    return a.tolist(), t.tolist()


@pytest.mark.parametrize("V", [65537, 70001, 128256])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("sampled", [True, False])
def test_workspaces_of_any_contents(dtype, sampled, V):
    """Rows that start on any element; sums of another call, NaN and huge ones left behind."""
    B, g = 3, 2
    p, q, draft, u = make(B, g, V, dtype, V % 11, sampled)
    flat = torch.empty(p.numel() + 1, dtype=p.dtype, device=DEV)
    flat[1:] = p.flatten()
    n = need(B, g, V)
    for fill in (0, 0x7F, 255):
        print(f"[spec, workspace of {fill}] {dtype}, {V}", flush=True)
        ws = torch.full((n + 64,), fill, dtype=torch.uint8, device=DEV)
        check(flat[1:].view(p.shape), q, draft, u, workspace=ws)
        assert bool((ws[n:] == fill).all())  # no more of it than the query says
        check(*make(B, g, V, dtype, fill + 1, sampled), workspace=ws)  # over the last call's sums


@pytest.mark.parametrize("V", [70001, 128256])
def test_streams(V):
    p, q, draft, u = make(8, 4, V, "f32", 3)
    want = check(p, q, draft, u)
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    got = [md.md_spec_accept(p, q, draft, u, stream=s) for s in (a, b) * 4]
    torch.cuda.synchronize()
    for acc, tok in got:
        assert torch.equal(acc, want[0]) and torch.equal(tok, want[1])


@pytest.mark.parametrize("V,dtype,sampled", [(70001, "bf16", False), (128256, "f32", True)])
def test_two_graphs_over_one_workspace(V, dtype, sampled):
    """Two captured calls of different batches share a workspace and are replayed in turn, with
    new inputs in the same buffers and eager calls in between: no sum or count of the other call
    or of the last replay shows."""
    g = 3
    cases = [(6, make(6, g, V, dtype, 1, sampled), outputs(6, g)),
             (2, make(2, g, V, dtype, 2, sampled), outputs(2, g))]
    ws = torch.full((max(need(B, g, V) for B, _, _ in cases),), 255, dtype=torch.uint8, device=DEV)
    graphs = []
    for _, x, (acc, tok) in cases:
        md.md_spec_accept(*x, accepted=acc, tokens=tok, workspace=ws)  # the first call, eager
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            md.md_spec_accept(*x, accepted=acc, tokens=tok, workspace=ws)
        graphs.append(graph)
    for seed in range(3, 7):
        print(f"[spec, two graphs] {dtype}, {V}, seed {seed}", flush=True)
        want = []
        for B, x, _ in cases:
            for old, new in zip(x, make(B, g, V, dtype, seed + B, sampled)):
                if old is not None:
                    old.copy_(new)
            want.append(reference(*x))
        for graph in graphs + graphs[::-1]:
            graph.replay()
        torch.cuda.synchronize()
        for (_, x, (acc, tok)), (a, t) in zip(cases, want):
            assert acc.tolist() == a and tok.tolist() == t
            check(*x)  # the program's own eager call
        ws.fill_(0x7F)
        torch.cuda.synchronize()


def test_every_segment_is_drawn_from():
    """u on a grid over two-launch rows whose mass sits in one token a segment, exactly: each
    draw is that segment's token."""
    V, seg = 128256, 1024
    n = -(-V // seg)
    at = np.minimum(np.arange(n) * seg + (np.arange(n) * 37) % seg, V - 1)
    p = torch.zeros((n, 1, V), device=DEV)
    p[:, :, torch.from_numpy(at).to(DEV)] = 2.0 ** -7
    u = ((torch.arange(n, dtype=torch.float64) + 0.5) / n).float().to(DEV)[:, None]
    assert need(n, 0, V)
    _, tok = check(p, None, torch.empty((n, 0), dtype=torch.int32, device=DEV), u)
    assert tok[:, 0].tolist() == at.tolist()
