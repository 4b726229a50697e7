"""The 4-bit attention's instances and plans on the GPU, against float64: every number of row
tiles, whole and cut; long runs of tiles in one wave, where page ids are refilled and the
running maximum moves; windows under ranges.  Each test asserts the plan it is about from the
workspace query."""
import numpy as np
import pytest
import torch

import kv4_reference
import paper_2408_11049_amd as md
import plain_ops as plain

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
TILE = 32                    # tokens of a step of a wave
WAVES = 4                    # of a workgroup, which take a unit's tiles in turn
REFILL = 32                  # tiles of a wave that one load of page ids serves


def say(text):
    print(text, flush=True)


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def queries(B, L, Hq, d, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randn((B, L, Hq, d), generator=g).to(DT[dtype]).to(DEV)


def pool(blocks, toks, Hkv, d, seed):
    """Blocks of random rows, no two alike; scales around one."""
    g = torch.Generator(DEV).manual_seed(seed)
    c = md.kv4_empty(blocks, toks, Hkv, d, device=DEV)
    for t, lo, hi in ((c.k, 0, 256), (c.v, 0, 256), (c.k_scale, 124, 128), (c.v_scale, 124, 128)):
        t.copy_(torch.randint(lo, hi, t.shape, generator=g, dtype=torch.uint8, device=DEV))
    return c


def tables(B, cols, blocks, seed):
    """Pages of the pool for every sequence, which share them in orders of their own."""
    rng = np.random.default_rng(seed)
    return ints(np.stack([np.resize(rng.permutation(blocks), cols) for _ in range(B)]).tolist())


def made(lens, Hkv, d, page, seed):
    cap = max(lens)
    if not page:
        return pool(len(lens), cap, Hkv, d, seed), None
    cols = -(-cap // page)
    blocks = cols + 5
    return pool(blocks, page, Hkv, d, seed), tables(len(lens), cols, blocks, seed)


def need(q, cache, pt, lens, n_sink=0, window=None):
    mode = dict(mode=md.MD_MODE_DRAFT, n_sink=n_sink, window=window) if window else {}
    return md.md_kv4_workspace_bytes(q, cache, ints(lens), page_table=pt, max_kv_len=max(lens), **mode)


def check(q, cache, pt, lens, dtype, n_sink=0, window=None, scale=0.0):
    out = torch.full_like(q, float("nan"))
    lse = torch.full(q.shape[:3], float("nan"), dtype=torch.float32, device=DEV)
    kw = dict(page_table=pt, out=out, lse=lse, sm_scale=scale, max_kv_len=max(max(lens), q.shape[1]))
    if window is None:
        md.md_kv4_verify_attn(q, cache, ints(lens), **kw)
    else:
        md.md_kv4_draft_attn(q, cache, ints(lens), n_sink, window, **kw)
    torch.cuda.synchronize()
    ro, rl, mass, qk, vmax = kv4_reference.attention(q, cache, pt, lens, n_sink, window,
                                                     scale or None)
    ob, lb = plain.attention_bounds(dtype, max(lens), ro, rl, mass, qk, q.shape[3], vmax)
    go, gl = out.double().cpu().numpy(), lse.double().cpu().numpy()
    fin = np.isfinite(rl)
    assert np.array_equal(fin, np.isfinite(gl)) and (gl[~fin] == -np.inf).all()
    worst = np.max(np.abs(go - ro) / np.maximum(ob, 1e-300))
    assert (np.abs(go - ro) <= ob).all(), f"O {worst:.2f} times its bound off"
    assert (np.abs(gl[fin] - rl[fin]) <= lb[fin]).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("Hq,Hkv,L", [(8, 2, 5), (11, 1, 3), (16, 2, 5), (12, 1, 4), (14, 2, 7),
                                      (16, 2, 8)])
def test_row_tiles_whole_and_cut(Hq, Hkv, L, page, d):
    """bf16 units of 20, 33, 40, 48, 49 and 64 rows (two to four row tiles), as a workgroup each
    and cut into many pieces."""
    for lens in ([1, L, 31, 33, 0, 200, 64], [2600, 40, 0, 5003, L]):
        say(f"[row tiles] {Hq} on {Hkv}, {L} tokens, d {d}, page {page}, lengths {lens}")
        cache, pt = made(lens, Hkv, d, page, Hq + L)
        q = queries(len(lens), L, Hq, d, "bf16", L)
        assert (need(q, cache, pt, lens) > 0) == (max(lens) > 1000)
        check(q, cache, pt, lens, "bf16")


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("dtype,d,Hq,L,scale", [("bf16", 128, 2, 2, 0.0), ("bf16", 64, 8, 5, 0.6),
                                                ("f32", 128, 4, 3, 0.6)])
@pytest.mark.parametrize("window", [None, 8500])
def test_long_runs_of_whole_units(dtype, d, Hq, L, scale, page, window):
    """More sequences than ranges are made for: a unit is a workgroup's at any length, here 282
    tiles, 70 for each wave, which takes three loads of page ids.  With a scale of 0.6 the maximum
    moves on the way."""
    lens = [9001, 8877] + [5, 0, 33] * 341
    assert len(lens) == 1025 and 8877 // TILE // WAVES > 2 * REFILL
    say(f"[long runs, whole] {dtype}, d {d}, {Hq} heads, {L} tokens, page {page}, window {window}")
    cache, pt = made(lens, 1, d, page, page)
    q = queries(len(lens), L, Hq, d, dtype, 3)
    assert need(q, cache, pt, lens, 70 if window else 0, window) == 0
    check(q, cache, pt, lens, dtype, 70 if window else 0, window, scale)


@pytest.mark.parametrize("dtype,d,Hq,L,page,B,scale", [
    ("bf16", 128, 64, 5, 16, 20, 0.0),   # 40 rows: three row tiles
    ("bf16", 128, 32, 5, 64, 32, 0.6),   # 20 rows
    ("bf16", 64, 16, 2, 16, 40, 0.6), ("f32", 128, 16, 3, 16, 32, 0.0),
    ("f32", 128, 64, 5, 64, 14, 0.0)])   # two passes over a head's K and V
def test_long_runs_of_ranges(dtype, d, Hq, L, page, B, scale):
    """Ranges of more than 128 tiles that begin anywhere in a unit and end in the next: more
    than 32 for each wave."""
    lens = np.random.default_rng(B).integers(9000, 26000, B).tolist()
    lens[3], lens[7] = 0, 17
    lens[1] = 30011
    say(f"[long runs, ranges] {dtype}, d {d}, {Hq} heads, {L} tokens, page {page}, {B} sequences")
    cache, pt = made(lens, 8, d, page, B)
    q = queries(B, L, Hq, d, dtype, 4)
    R = Hq // 8 * L
    NT = min(-(-R // 16), 4 if dtype == "bf16" else 2)
    passes = -(-R // (16 * NT)) if dtype == "f32" else 1
    # A workgroup's share of the workspace: two partial results (rows of O, maximum and sum).
    workgroups = need(q, cache, pt, lens) // (2 * 16 * NT * (d + 2) * 4)
    tiles = sum(max(-(-n // TILE), 1) for n in lens) * 8 * passes
    say(f"  {workgroups} workgroups, {tiles} tiles: {tiles / max(workgroups, 1):.0f}")
    assert 0 < workgroups and tiles // workgroups > WAVES * REFILL
    check(q, cache, pt, lens, dtype, scale=scale)


@pytest.mark.parametrize("dtype,d,Hq,L", [("bf16", 128, 8, 1), ("bf16", 64, 16, 5), ("f32", 128, 4, 3)])
@pytest.mark.parametrize("page", [0, 4, 16, 64])
@pytest.mark.parametrize("n_sink,window", [(0, 3000), (5, 3000), (70, 3001), (2000, 1), (33, 8000)])
def test_windows_under_ranges(dtype, d, Hq, L, page, n_sink, window):
    """Pieces on either side of the gap between sinks and window, and across it."""
    lens = [9000, 6500, 3100, 20, 0, 4097, 8031]
    say(f"[windows, ranges] {dtype}, d {d}, {L} tokens, page {page}, {n_sink} + {window}")
    cache, pt = made(lens, 2, d, page, page + 1)
    q = queries(len(lens), L, Hq, d, dtype, 5)
    assert need(q, cache, pt, lens, n_sink, window) > 0
    check(q, cache, pt, lens, dtype, n_sink, window)


def test_two_graphs_over_one_workspace():
    """A verify and a draft, captured over one workspace, replayed in turn with new lengths and
    eager calls between: no partial result or join of the other shows."""
    lens, B, L, Hkv, d = ints([7000, 40, 3333, 5100]), 4, 2, 2, 128
    cache, pt = made([7000] * B, Hkv, d, 16, 9)
    q = queries(B, L, 8, d, "bf16", 9)
    top = dict(page_table=pt, max_kv_len=7000)
    mode = dict(mode=md.MD_MODE_DRAFT, n_sink=5, window=3000)
    sizes = [md.md_kv4_workspace_bytes(q, cache, lens, **top),
             md.md_kv4_workspace_bytes(q, cache, lens, **top, **mode)]
    assert min(sizes) > 0
    ws = torch.full((max(sizes),), 255, dtype=torch.uint8, device=DEV)

    def verify(**kw):
        return md.md_kv4_verify_attn(q, cache, lens, **top, **kw)

    def draft(**kw):
        return md.md_kv4_draft_attn(q, cache, lens, 5, 3000, **top, **kw)
    graphs, outs = [], []
    for f in (verify, draft):
        o, lse = f()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            f(out=o, lse=lse, workspace=ws)
        graphs.append(graph)
        outs.append((o, lse))
    for ends in ([7000, 40, 3333, 5100], [1, 6999, 0, 64], [5100, 5100, 5100, 5100], [33, 7000, 7000, 2]):
        say(f"[two graphs] {ends}")
        lens.copy_(ints(ends))
        want = [f() for f in (verify, draft)]
        for graph in graphs + graphs[::-1]:
            graph.replay()
        torch.cuda.synchronize()
        for (o, lse), (wo, wl) in zip(outs, want):
            assert torch.equal(o, wo) and torch.equal(lse, wl)
        check(q, cache, pt, ends, "bf16")
        check(q, cache, pt, ends, "bf16", 5, 3000)
