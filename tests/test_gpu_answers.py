"""Attention over a shared prefix, accumulated weights, eviction and token log probabilities
on the GPU, against float64 formulas."""
import numpy as np
import pytest
import torch

import paper_2408_11049_amd as md
import plain_answers as plain

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def host(t):
    return t.detach().to(torch.float64).cpu().numpy()


def rand(gen, shape, dt, scale=1.0):
    return (torch.randn(shape, generator=gen) * scale).to(DT[dt]).to(DEV)


class Cache:
    """K and V of `n` sequences of up to `cap` tokens, contiguous or paged, with NaN in every place
    that no token holds."""

    def __init__(self, gen, lens, cap, Hkv, d, dt, page=0, heads_first=False, spare=1):
        n = len(lens)
        self.lens_np, self.page = np.asarray(lens), page
        rows = [[torch.randn((int(s), Hkv, d), generator=gen).to(DT[dt]) for s in lens] for _ in "kv"]
        self.rows = [[host(r) for r in x] for x in rows]
        if page:
            cols = max(1, -(-cap // page))
            blocks, toks = n * cols + spare, page
            perm = torch.randperm(blocks, generator=gen)[: n * cols].reshape(n, cols)
            self.table = perm.to(torch.int32).to(DEV)
        else:
            blocks, toks, self.table = n, max(cap, 1), None
        shape = (blocks, Hkv, toks, d) if heads_first else (blocks, toks, Hkv, d)
        self.k, self.v = (torch.full(shape, float("nan"), dtype=DT[dt]) for _ in "kv")
        if heads_first:
            self.k, self.v = self.k.transpose(1, 2), self.v.transpose(1, 2)
        for t, x in ((self.k, rows[0]), (self.v, rows[1])):
            for b, r in enumerate(x):
                for c in range(-(-len(r) // page) if page else 1):
                    if page:
                        part = r[c * page:(c + 1) * page]
                        t[perm[b, c], : len(part)] = part
                    else:
                        t[b, : len(r)] = r
        if heads_first:  # keep the layout on the device
            self.k, self.v = (t.transpose(1, 2).contiguous().to(DEV).transpose(1, 2) for t in (self.k, self.v))
        else:
            self.k, self.v = self.k.to(DEV), self.v.to(DEV)
        self.lens = torch.tensor(list(lens), dtype=torch.int32, device=DEV)
        self.cap = toks if not page else self.table.shape[1] * page


def check_prefix(dt, Hq, Hkv, d, L, lens, plens, page=0, ppage=0, heads_first=False, scale=0.0, seed=0,
                 **kw):
    gen = torch.Generator().manual_seed(seed)
    own = Cache(gen, lens, max(max(lens), L), Hkv, d, dt, page, heads_first)
    pre = Cache(gen, plens, max(plens), Hkv, d, dt, ppage, heads_first)
    q = rand(gen, (len(lens), L, Hq, d), dt)
    out = torch.full_like(q, float("nan"))
    lse = torch.full(q.shape[:3], float("nan"), device=DEV)
    md.md_prefix_attn(q, own.k, own.v, own.lens, pre.k, pre.v, pre.lens, page_table=own.table,
                      prefix_page_table=pre.table, out=out, lse=lse, sm_scale=scale, **kw)
    ro, rl, mass, qk = plain.prefix_attention(host(q), *own.rows, lens, *pre.rows, plens, scale or None)
    n = max(lens) + max(plens)
    top = max([float(np.abs(r).max()) for r in own.rows[1] + pre.rows[1] if r.size] + [0.0])
    ob, lb = plain.prefix_bounds(dt, n, ro, rl, mass, qk, d, top)
    none = np.isinf(rl)
    assert np.array_equal(np.isinf(host(lse)), none) and (host(out)[none] == 0).all()
    assert (np.abs(host(out) - ro) <= ob).all(), np.abs(host(out) - ro).max()
    assert (np.abs(host(lse)[~none] - rl[~none]) <= lb[~none]).all()


PREFIX = [
    # Hq, Hkv, d, L, own lengths, prefix lengths, page, prefix page
    ("bf16", 8, 2, 128, 1, [1, 5], [200], 0, 0),
    ("bf16", 8, 2, 128, 4, [4, 9, 70, 200], [64, 65], 16, 16),
    ("bf16", 8, 1, 64, 2, [2, 3, 64, 65, 129, 17], [1, 63, 0], 16, 0),
    ("f32", 4, 1, 64, 4, [4, 40], [100], 0, 0),
    ("f32", 4, 2, 128, 3, [3, 31, 33, 200], [0, 97], 0, 64),
    ("f32", 12, 4, 64, 1, [1, 2, 3], [33, 32, 31], 16, 16),
    ("bf16", 7, 1, 128, 9, [9, 100], [130], 64, 16),          # 63 rows of a head
    ("bf16", 64, 8, 128, 8, [8, 20], [10], 0, 0),             # 64
    ("bf16", 4, 1, 128, 1, [3] * 40, [300], 0, 16),           # 160 rows of a prefix: two blocks
    ("bf16", 4, 1, 64, 5, [5 + 3 * i for i in range(13)], [1000], 16, 16),  # 260 rows
    ("f32", 4, 1, 128, 2, [2 + i for i in range(17)], [70], 0, 0),          # 136 rows
    ("bf16", 3, 3, 128, 1, [1] * 5, [1], 0, 0),               # one key each
    ("bf16", 32, 8, 128, 1, [300, 1, 17, 64], [2000], 16, 16),
]


@pytest.mark.parametrize("case", PREFIX, ids=[str(i) for i in range(len(PREFIX))])
def test_prefix_attention(case):
    check_prefix(*case)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_prefix_heads_first_layout_and_scale(dt):
    check_prefix(dt, 8, 2, 64, 2, [2, 77, 5, 9], [90, 130], heads_first=True, scale=0.3)
    check_prefix(dt, 8, 2, 128, 2, [2, 77], [90], 16, 64, heads_first=True, scale=0.02)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_rows_that_see_the_prefix_alone_or_nothing(dt):
    """Fewer own tokens than rows: the first rows see the prefix only, and nothing where it is
    empty."""
    check_prefix(dt, 4, 1, 64, 4, [0, 2, 4, 1], [0, 50])
    check_prefix(dt, 4, 2, 128, 3, [0, 1], [0])


def test_no_prefix_at_all():
    """max_prefix_len 0: the own caches alone."""
    gen = torch.Generator().manual_seed(3)
    own = Cache(gen, [5, 90], 90, 2, 64, "bf16")
    q = rand(gen, (2, 2, 4, 64), "bf16")
    empty = torch.empty((1, 0, 2, 64), dtype=torch.bfloat16, device=DEV)
    zero = torch.zeros(1, dtype=torch.int32, device=DEV)
    o, lse = md.md_prefix_attn(q, own.k, own.v, own.lens, empty, empty, zero)
    ro, rl, mass, qk = plain.prefix_attention(host(q), *own.rows, [5, 90], [np.zeros((0, 2, 64))],
                                              [np.zeros((0, 2, 64))], [0])
    ob, lb = plain.prefix_bounds("bf16", 90, ro, rl, mass, qk, 64, 6.0)
    assert (np.abs(host(o) - ro) <= ob).all() and (np.abs(host(lse) - rl) <= lb).all()


def test_scores_of_growing_size():
    """Keys whose scores rise along the prefix: the running maximum moves in every tile."""
    gen = torch.Generator().manual_seed(4)
    d, T = 64, 700
    pk = (torch.arange(T)[:, None, None] / 40.0 * torch.ones((T, 1, d))).to(torch.bfloat16)
    pv = torch.randn((T, 1, d), generator=gen).to(torch.bfloat16)
    own = Cache(gen, [3, 3], 3, 1, d, "bf16")
    q = (torch.ones((2, 1, 4, d)) * 0.5).to(torch.bfloat16).to(DEV)
    lens = torch.tensor([T], dtype=torch.int32, device=DEV)
    o, lse = md.md_prefix_attn(q, own.k, own.v, own.lens, pk[None].to(DEV), pv[None].to(DEV), lens)
    ro, rl, mass, qk = plain.prefix_attention(host(q), *own.rows, [3, 3], [host(pk)], [host(pv)], [T])
    ob, lb = plain.prefix_bounds("bf16", T, ro, rl, mass, qk, d, 6.0)
    assert (np.abs(host(o) - ro) <= ob).all() and (np.abs(host(lse) - rl) <= lb).all()


def test_infinities_and_nan_reach_their_rows_only():
    """An own key of NaN makes its sequence's later rows NaN (lse -inf), and no other; a key of
    -inf for one channel that the query holds positive is no key at all."""
    gen = torch.Generator().manual_seed(5)
    own = Cache(gen, [6, 6, 6, 6], 6, 1, 64, "bf16")
    pre = Cache(gen, [100], 100, 1, 64, "bf16")
    q = rand(gen, (4, 2, 4, 64), "bf16").abs()
    clean, _ = md.md_prefix_attn(q, own.k, own.v, own.lens, pre.k, pre.v, pre.lens)
    k = own.k.clone()
    k[1, 5, 0, 3] = float("nan")    # seen by the second row alone
    k[2, 0, 0] = 0.0
    k[2, 0, 0, 7] = float("-inf")
    o, lse = md.md_prefix_attn(q, k, own.v, own.lens, pre.k, pre.v, pre.lens)
    assert torch.equal(o[0], clean[0]) and torch.equal(o[3], clean[3]) and torch.equal(o[1, 0], clean[1, 0])
    assert o[1, 1].isnan().all() and (lse[1, 1] == float("-inf")).all()
    assert torch.isfinite(o[2].float()).all()
    want = plain.prefix_attention(host(q[2:3]), [own.rows[0][2][1:]], [own.rows[1][2][1:]], [5],
                                  *pre.rows, [100])[0]
    assert np.abs(host(o[2]) - want[0]).max() < 2e-2


def test_error_word_reports_both_caches():
    gen = torch.Generator().manual_seed(6)
    own = Cache(gen, [20, 20], 20, 1, 64, "bf16", 16)
    pre = Cache(gen, [40], 40, 1, 64, "bf16", 16)
    q = rand(gen, (2, 2, 4, 64), "bf16")

    def bits(**over):
        a = dict(kv_lens=own.lens, prefix_lens=pre.lens, page_table=own.table,
                 prefix_page_table=pre.table)
        a.update(over)
        word = torch.zeros(1, dtype=torch.int32, device=DEV)
        md.md_prefix_attn(q, own.k, own.v, a["kv_lens"], pre.k, pre.v, a["prefix_lens"],
                          page_table=a["page_table"], prefix_page_table=a["prefix_page_table"],
                          max_kv_len=20, max_prefix_len=40, err_word=word)
        return int(word)

    def ints(*x):
        return torch.tensor(x, dtype=torch.int32, device=DEV)
    assert bits() == 0
    assert bits(kv_lens=ints(20, 1)) == md.MD_ERRW_SHORT_LEN
    assert bits(kv_lens=ints(21, 20)) == md.MD_ERRW_LONG_LEN
    assert bits(prefix_lens=ints(41)) == md.MD_ERRW_LONG_LEN
    assert bits(prefix_lens=ints(-1)) == md.MD_ERRW_SHORT_LEN
    bad = own.table.clone()
    bad[1, 1] = own.k.shape[0]
    assert bits(page_table=bad) == md.MD_ERRW_BAD_PAGE
    bad = pre.table.clone()
    bad[0, 0] = -1
    assert bits(prefix_page_table=bad) == md.MD_ERRW_BAD_PAGE


# ---- accumulated weights ----

def row_lse(q, k, lens, scale=None):
    """float64 lse of the attention over the own cache, and its rounding to fp32."""
    z = [np.zeros((0,) + k[0].shape[1:])] * 1
    lse = plain.prefix_attention(q, k, k, lens, z, z, [0], scale)[1]
    return lse.astype(np.float32)


MASS = [
    # dt, Hq, Hkv, d, L, lengths, page, accepted
    ("bf16", 8, 2, 128, 1, [1, 2, 130], 0, False),
    ("bf16", 8, 2, 64, 5, [5, 127, 128, 129, 260], 16, True),
    ("f32", 4, 1, 64, 4, [4, 33, 200], 0, True),
    ("f32", 4, 2, 128, 3, [3, 300], 64, False),
    ("bf16", 21, 3, 128, 7, [7, 150], 16, True),     # 49 rows: a tile and a part of one
    ("bf16", 4, 4, 64, 1, [400], 0, False),
    ("bf16", 8, 2, 128, 200, [200, 230], 0, False),  # a prompt whole, and one after 30 tokens
    ("f32", 8, 4, 64, 130, [130], 16, False),
    ("bf16", 64, 8, 128, 20, [20, 41], 0, True),     # 160 rows
]


@pytest.mark.parametrize("case", MASS, ids=[str(i) for i in range(len(MASS))])
@pytest.mark.parametrize("slots", [0, 13])
def test_mass(case, slots):
    dt, Hq, Hkv, d, L, lens, page, part = case
    gen = torch.Generator().manual_seed(len(lens) * 7 + L)
    c = Cache(gen, lens, max(lens), Hkv, d, dt, page)
    B, S = len(lens), max(lens) + slots
    q = rand(gen, (B, L, Hq, d), dt)
    lse = row_lse(host(q), c.rows[0], lens)
    acc = np.array([(3 * b) % L if b % 3 else L + 5 for b in range(B)]) if part else None
    mass = torch.rand((B, Hkv, S), generator=gen)
    pos = torch.randint(0, 999, (B, Hkv, S), generator=gen).to(torch.int32)
    pos0 = np.array([1000 * b + 17 for b in range(B)])
    m, x = mass.to(DEV), pos.to(DEV)
    got = md.md_kv_mass(q, c.k, c.lens, torch.from_numpy(lse).to(DEV), m, x,
                        torch.from_numpy(pos0.astype(np.int32)).to(DEV),
                        accepted=None if acc is None else torch.from_numpy(acc.astype(np.int32)).to(DEV),
                        max_kv_len=max(lens), page_table=c.table)
    assert got is m
    want, wpos, err = plain.kv_mass(host(q), c.rows[0], lens, lse.astype(np.float64), mass.numpy().astype(np.float64),
                                    pos.numpy(), pos0, acc)
    assert np.array_equal(x.cpu().numpy(), wpos)
    assert (np.abs(host(m) - want) <= err).all(), (np.abs(host(m) - want) - err).max()


def test_mass_of_a_whole_prompt_sums_to_its_rows():
    """Every row gives away a weight of one for each query head."""
    gen = torch.Generator().manual_seed(8)
    L, Hq, Hkv = 96, 4, 2
    c = Cache(gen, [L], L, Hkv, 64, "f32")
    q = rand(gen, (1, L, Hq, 64), "f32")
    lse = torch.from_numpy(row_lse(host(q), c.rows[0], [L])).to(DEV)
    m = torch.full((1, Hkv, L), float("nan"), device=DEV)
    x = torch.empty((1, Hkv, L), dtype=torch.int32, device=DEV)
    md.md_kv_mass(q, c.k, c.lens, lse, m, x, torch.zeros(1, dtype=torch.int32, device=DEV))
    assert torch.equal(x[0, 0], torch.arange(L, dtype=torch.int32, device=DEV))
    assert np.allclose(host(m).sum(2), L * Hq / Hkv, rtol=1e-5)


def test_mass_short_lengths_and_empty_rows():
    """Rows before the cache's first token weigh nothing, nor do rows of lse -inf; a length of 0
    leaves everything as it is."""
    gen = torch.Generator().manual_seed(9)
    lens, L = [0, 2, 5], 4
    c = Cache(gen, lens, 5, 1, 64, "bf16")
    q = rand(gen, (3, L, 4, 64), "bf16")
    lse = row_lse(host(q), c.rows[0], lens)
    lse[2, 1] = -np.inf
    mass, pos = np.ones((3, 1, 6)), np.full((3, 1, 6), -7)
    m = torch.ones((3, 1, 6), device=DEV)
    x = torch.full((3, 1, 6), -7, dtype=torch.int32, device=DEV)
    p0 = torch.tensor([4, 50, 60], dtype=torch.int32, device=DEV)
    md.md_kv_mass(q, c.k, c.lens, torch.from_numpy(lse).to(DEV), m, x, p0, max_kv_len=5)
    want, wpos, err = plain.kv_mass(host(q), c.rows[0], lens, lse.astype(np.float64), mass, pos, [4, 50, 60])
    assert np.array_equal(x.cpu().numpy(), wpos) and (np.abs(host(m) - want) <= err).all()


# ---- eviction ----

def check_evict(dt, Hkv, d, lens, slots, budget, n_sink=0, recent=0, page=0, masses=None, seed=0,
                heads_first=False):
    gen = torch.Generator().manual_seed(seed)
    B = len(lens)
    c = Cache(gen, [slots] * B, slots, Hkv, d, dt, page, heads_first)
    mass = torch.rand((B, Hkv, slots), generator=gen).numpy() if masses is None else masses(B, Hkv, slots)
    mass = mass.astype(np.float32)
    rng = np.random.default_rng(seed)
    seq = np.array([max(int(n), 0) + 50 for n in lens])
    pos = np.stack([np.stack([rng.permutation(slots + 50)[:slots] for _ in range(Hkv)]) for _ in range(B)])
    kb, vb = c.k.clone(), c.v.clone()
    m, x = torch.from_numpy(mass.copy()).to(DEV), torch.from_numpy(pos.astype(np.int32)).to(DEV)
    out = md.md_kv_evict(c.k, c.v, m, x, torch.tensor(lens, dtype=torch.int32, device=DEV),
                         torch.from_numpy(seq.astype(np.int32)).to(DEV), budget, n_sink=n_sink,
                         recent=recent, page_table=c.table)
    names = np.broadcast_to(np.arange(slots), mass.shape).copy()
    from_, wm, wx, wl = plain.evict(names, mass, pos, lens, seq, budget, n_sink, recent)
    assert np.array_equal(out.cpu().numpy(), wl)
    assert np.array_equal(m.cpu().numpy().view(np.int32), wm.view(np.int32))
    assert np.array_equal(x.cpu().numpy(), wx)

    def logical(t):
        t = t if c.table is None else t[c.table.long()].flatten(1, 2)
        return t[:, :slots].permute(0, 2, 1, 3)
    at = torch.from_numpy(from_).to(DEV)[..., None].expand(-1, -1, -1, d)
    for before, after in ((kb, c.k), (vb, c.v)):
        assert torch.equal(logical(after), logical(before).gather(2, at))
        if c.table is not None:                      # pages of no sequence stay as they were
            spare = [i for i in range(before.shape[0]) if i not in set(c.table.flatten().tolist())]
            assert torch.equal(after[spare].view(torch.uint8), before[spare].view(torch.uint8))
    return from_


EVICT = [
    # dt, Hkv, d, lens, slots, budget, n_sink, recent, page
    ("bf16", 2, 128, [20, 16, 17, 5, 0], 20, 16, 0, 0, 0),
    ("bf16", 3, 64, [40, 39], 40, 8, 2, 4, 16),
    ("f32", 1, 64, [300, 257, 256, 255], 300, 256, 4, 100, 0),
    ("f32", 2, 128, [70], 70, 1, 0, 0, 64),
    ("bf16", 1, 128, [1500, 900, 1100], 1500, 700, 16, 600, 16),   # moved by a launch of their own
    ("bf16", 2, 64, [5000, 4097], 5000, 900, 0, 0, 0),             # the wide workgroup
    ("bf16", 2, 64, [4500, 4100], 4500, 4090, 3, 4000, 16),
    ("bf16", 8, 128, [12] * 6, 12, 8, 1, 7, 0),                    # all kept are held
]


@pytest.mark.parametrize("case", EVICT, ids=[str(i) for i in range(len(EVICT))])
def test_evict(case):
    check_evict(*case)


def test_evict_weights_of_any_kind():
    """Ties, NaN, infinities, both zeros, negative weights and denormals order as documented."""
    def odd(B, Hkv, slots):
        rng = np.random.default_rng(1)
        pool = np.array([0.0, -0.0, 1.0, 1.0, np.nan, -np.nan, np.inf, -np.inf, -2.5, 1e-42, 3e38, -1e-45])
        return pool[rng.integers(0, len(pool), (B, Hkv, slots))]
    for budget in (1, 33, 60, 99):
        check_evict("bf16", 2, 64, [100, 90], 100, budget, masses=odd)
    check_evict("bf16", 1, 64, [700], 700, 640, masses=lambda *s: np.ones(s))
    check_evict("bf16", 1, 64, [5000], 5000, 1000, masses=lambda *s: np.zeros(s), heads_first=True)
    check_evict("f32", 2, 64, [64, 64], 64, 20, masses=lambda *s: np.full(s, np.nan), heads_first=True)


def test_evict_bad_pages_are_left_alone():
    """Rows on pages outside the pool are not touched; the bookkeeping goes on."""
    gen = torch.Generator().manual_seed(2)
    c = Cache(gen, [64], 64, 1, 64, "bf16", 16)
    table = c.table.clone()
    table[0, 1] = c.k.shape[0] + 3
    table[0, 3] = -2
    m = torch.arange(64, dtype=torch.float32, device=DEV)[None, None].contiguous()
    x = torch.zeros((1, 1, 64), dtype=torch.int32, device=DEV)
    k0 = c.k.clone()
    n = torch.tensor([64], dtype=torch.int32, device=DEV)
    out = md.md_kv_evict(c.k, c.v, m, x, n, n, 32, page_table=table)
    assert int(out[0]) == 32 and m[0, 0, :32].tolist() == list(range(32, 64))
    a, b = c.table[0, 0], c.table[0, 2]              # slots 0..15 take 32..47; the others are lost
    assert torch.equal(c.k[a], k0[b])
    for other in set(range(c.k.shape[0])) - {int(a)}:
        assert torch.equal(c.k[other].view(torch.uint8), k0[other].view(torch.uint8))


# ---- log probabilities ----

def check_logp(x, tokens, top_k, chunks=1):
    """x [.., V] on the device; tokens a host array or None."""
    flat = host(x).reshape(int(np.prod(x.shape[:-1])), x.shape[-1])
    t = None if tokens is None else torch.from_numpy(np.asarray(tokens).astype(np.int32)).reshape(x.shape[:-1]).to(DEV)
    lp, ent, top, tlp = md.md_token_logprobs(x, t, top_k=top_k)
    wlp, went, wtop, wtlp, lz = plain.token_logprobs(flat, None if t is None else np.asarray(tokens).reshape(-1), top_k)
    assert top.shape == x.shape[:-1] + (top_k,) and tlp.shape == top.shape and ent.shape == x.shape[:-1]
    assert np.array_equal(top.cpu().numpy().reshape(len(flat), top_k), wtop)
    with np.errstate(invalid="ignore"):
        size = np.nan_to_num(np.abs(np.where(np.isfinite(flat), flat, 0)).max(1)) + lz
        pairs = [(host(tlp).reshape(len(flat), top_k), wtlp, size[:, None])]
        if t is None:
            assert lp is None
        else:
            pairs.append((host(lp).reshape(-1), wlp, size))
        for got, want, s in pairs:
            assert np.array_equal(np.isnan(got), np.isnan(want))
            assert np.array_equal(np.isneginf(got), np.isneginf(want))
            ok = np.isfinite(want)
            err, lim = np.abs(got - want), np.broadcast_to(plain.logprob_bound(np.where(ok, want, 0), s, chunks), want.shape)
            assert (err[ok] <= lim[ok]).all(), (err[ok] - lim[ok]).max()
        got = host(ent).reshape(-1)
        assert np.array_equal(np.isnan(got), np.isnan(went))
        ok = np.isfinite(went)
        # ln z - t / z: both terms as a log probability, t's by its own size (ln z and the entropy).
        lim = plain.logprob_bound(0, lz, chunks) * (2 + 2 * np.abs(lz) + 2 * np.abs(went))
        assert (np.abs(got - went)[ok] <= lim[ok]).all()


LOGP = [
    # rows, vocab, dt, top_k
    ((1,), 1, "f32", 1), ((2, 3), 5, "bf16", 8), ((3,), 63, "f32", 32), ((2,), 1000, "bf16", 5),
    ((5,), 4096, "f32", 20), ((1,), 4097, "bf16", 32), ((2, 2), 4101, "f32", 0), ((3,), 16385, "bf16", 7),
    ((1,), 50001, "bf16", 5), ((1,), 50001, "f32", 32), ((300,), 16384, "f32", 3), ((260,), 17003, "bf16", 20),
    ((64, 5), 33000, "f32", 20), ((2,), 128256, "f32", 20), ((0,), 100, "f32", 4),
]


@pytest.mark.parametrize("case", LOGP, ids=[f"{c[0]}x{c[1]}-{c[2]}-{c[3]}" for c in LOGP])
def test_logprobs(case):
    lead, V, dt, K = case
    gen = torch.Generator().manual_seed(V + K)
    x = rand(gen, lead + (V,), dt, 3.0)
    n = int(np.prod(lead))
    tok = torch.randint(-1, V + 1, (n,), generator=gen).numpy().reshape(lead)  # none, and past the end
    check_logp(x, tok, K)
    check_logp(x, None, K)


def test_logprobs_of_clustered_rows():
    """Equal, ascending and descending values, and all the largest ones in one lane."""
    V = 20000
    rows = [np.full(V, 2.5), np.arange(V) / 500.0, -np.arange(V) / 500.0, np.tile([1.0, 1.0, 0.0], V)[:V],
            np.where(np.arange(V) % 256 < 4, 9.0, np.arange(V) % 7), (np.arange(V) // 64) % 11,
            np.where(np.arange(V) >= V - 600, 3.0, 0.0)]
    for dt in ("f32", "bf16"):
        x = torch.from_numpy(np.stack(rows)).to(DT[dt]).to(DEV)
        for K in (1, 20, 32):
            check_logp(x, np.arange(len(rows)) * 5, K)
        wide = x.repeat(40, 1)  # enough rows for 64 logits a lane
        check_logp(wide, np.arange(len(wide)), 20)


def test_logprobs_of_masked_rows():
    """-inf, the type's lowest value, NaN, +inf and rows of nothing."""
    V = 9000
    inf, low = np.inf, float(torch.finfo(torch.float32).min)
    base = np.random.default_rng(3).standard_normal(V) * 2
    few = np.full(V, -inf)
    few[[17, 4000, 8999]] = [1.0, 3.0, 1.0]
    lowest = np.full(V, low)
    lowest[[5, 6000]] = [2.0, -1.0]
    nan = base.copy()
    nan[77] = np.nan
    big = base.copy()
    big[5000] = inf
    nans = np.full(V, np.nan)
    mixed = np.full(V, -inf)
    mixed[100] = np.nan
    half = np.where(np.arange(V) < 5000, -inf, base)
    rows = np.stack([few, np.full(V, -inf), lowest, nan, big, nans, mixed, half, np.full(V, low),
                     base + 1000, base - 1000])
    tok = np.array([4000, 3, 5, 77, 5000, 0, 100, 10, 4, 8, 9])
    for K in (0, 1, 5, 32):
        check_logp(torch.from_numpy(rows).float().to(DEV), tok, K)
        check_logp(torch.from_numpy(rows[[0, 1, 4, 5, 6, 7]]).to(torch.bfloat16).to(DEV), tok[:6], K)
    check_logp(torch.from_numpy(np.tile(rows, (30, 2))).float().to(DEV), np.tile(tok, 30), 20)


def test_logprobs_of_strided_rows():
    """A vocabulary padded in memory, rows of every alignment, and every second row."""
    gen = torch.Generator().manual_seed(11)
    for dt in ("f32", "bf16"):
        x = rand(gen, (6, 5003), dt)
        tok = np.arange(6) * 100
        check_logp(x[:, :4999], tok, 4)
        check_logp(x[::2, 1:4200], tok[:3], 4)
        check_logp(x.view(2, 3, 5003)[:, :, 3:4099], tok, 4)
    with pytest.raises(ValueError, match="one stride"):
        md.md_token_logprobs(x.view(2, 3, 5003)[:, :2], top_k=1)
    with pytest.raises(ValueError, match="unit-stride"):
        md.md_token_logprobs(x.t(), top_k=1)
