"""Several answers of one prompt as a server runs them, on the GPU: the shared prefix, the step's weights, the
acceptance, the eviction and the tokens' log probabilities, eagerly, as a HIP graph, on other streams, with
workspaces of any contents, and at offsets past 32 bits."""
import numpy as np
import pytest
import torch

import paper_2408_11049_amd as md
import plain_answers as plain
from test_answers_binding import BAD_ON_GPU, host_call
from test_gpu_answers import DEV, Cache, check_evict, check_logp, check_prefix, host, rand, row_lse

pytestmark = pytest.mark.gpu
I32 = torch.int32


def ints(x):
    return torch.tensor(np.asarray(x), dtype=I32, device=DEV)


class Server:
    """B sequences over one prefix of T tokens, P prefixes in all, caches cut to `budget` tokens after each
    step of L.  Keeps every row ever appended, by its position, to say what a cache must hold."""

    def __init__(self, B=6, P=2, T=150, L=3, Hq=8, Hkv=2, d=64, budget=24, vocab=5000, page=16, seed=0):
        gen = torch.Generator().manual_seed(seed)
        self.B, self.L, self.Hq, self.Hkv, self.d, self.budget, self.vocab = B, L, Hq, Hkv, d, budget, vocab
        self.gen, self.slots = gen, budget + L
        self.pre = Cache(gen, [T, T - 30][:P], T, Hkv, d, "bf16", page)
        cols = -(-self.slots // page)
        self.table = torch.randperm(B * cols, generator=gen).reshape(B, cols).to(I32).to(DEV)
        self.k = torch.zeros((B * cols, page, Hkv, d), dtype=torch.bfloat16, device=DEV)
        self.v = torch.zeros_like(self.k)
        self.mass = torch.zeros((B, Hkv, self.slots), device=DEV)
        self.pos = torch.full((B, Hkv, self.slots), -1, dtype=I32, device=DEV)
        self.lens, self.seq, self.kv_lens = (torch.zeros(B, dtype=I32, device=DEV) for _ in range(3))
        self.before = torch.zeros(B, dtype=I32, device=DEV)
        self.acc = torch.zeros(B, dtype=I32, device=DEV)
        self.q = rand(gen, (B, L, Hq, d), "bf16")
        self.k_new, self.v_new = (rand(gen, (B, L, Hkv, d), "bf16") for _ in "kv")
        self.logits = rand(gen, (B, L, vocab), "bf16", 2.0)
        self.draft = torch.zeros((B, L - 1), dtype=I32, device=DEV)
        self.tokens = torch.zeros((B, L), dtype=I32, device=DEV)
        self.o = torch.empty_like(self.q)
        self.lse = torch.empty((B, L, Hq), device=DEV)
        self.lp, self.ent = (torch.empty((B, L), device=DEV) for _ in range(2))
        self.top, self.tlp = torch.empty((B, L, 5), dtype=I32, device=DEV), torch.empty((B, L, 5), device=DEV)
        n = md.md_prefix_workspace_bytes(self.q, self.k, self.v, self.kv_lens, self.pre.k, self.pre.v, self.pre.lens,
                                         page_table=self.table, prefix_page_table=self.pre.table, max_kv_len=self.slots)
        lib = md.load_library()
        n = max(n, lib.md_token_logprobs_workspace_bytes(B * L, vocab, 5),
                lib.md_greedy_accept_workspace_bytes(B, L - 1, vocab))
        self.ws = torch.full((n,), 255, dtype=torch.uint8, device=DEV)   # one for all: they run in turn
        self.history = [{} for _ in range(B)]

    def inputs(self):
        """The next step's: fresh rows, and drafts of which some are what the target takes."""
        for t in (self.q, self.k_new, self.v_new):
            t.copy_(rand(self.gen, t.shape, "bf16"))
        self.logits.copy_(rand(self.gen, self.logits.shape, "bf16", 2.0))
        best = self.logits.float().argmax(-1)[:, :-1].to(I32)
        wrong = (torch.rand(best.shape, generator=self.gen) < 0.4).to(DEV)
        self.draft.copy_(torch.where(wrong, (best + 1) % self.vocab, best))

    def step(self):
        md.md_kv_append(self.k, self.v, self.k_new, self.v_new, self.lens, page_table=self.table, lens_out=self.kv_lens)
        md.md_prefix_attn(self.q, self.k, self.v, self.kv_lens, self.pre.k, self.pre.v, self.pre.lens,
                          page_table=self.table, prefix_page_table=self.pre.table, max_kv_len=self.slots,
                          out=self.o, lse=self.lse, workspace=self.ws)
        md.md_greedy_accept(self.logits, self.draft, accepted=self.acc, tokens=self.tokens, want_target=False,
                            workspace=self.ws)
        md.md_token_logprobs(self.logits, self.tokens, top_k=5, logprobs=self.lp, entropy=self.ent, top=self.top,
                             top_logprobs=self.tlp, workspace=self.ws)
        md.md_kv_mass(self.q, self.k, self.kv_lens, self.lse, self.mass, self.pos, self.seq, accepted=self.acc,
                      max_kv_len=self.slots, page_table=self.table)
        md.md_kv_commit(self.lens, self.acc, self.L)
        md.md_kv_commit(self.seq, self.acc, self.L)
        self.before.copy_(self.lens)
        md.md_kv_evict(self.k, self.v, self.mass, self.pos, self.before, self.seq, self.budget, n_sink=2, recent=6,
                       page_table=self.table, lens_out=self.lens)

    STATE = ("k", "v", "mass", "pos", "lens", "seq", "kv_lens", "before", "acc", "tokens", "o", "lse", "lp", "ent",
             "top", "tlp")

    def state(self):
        return {n: getattr(self, n).clone() for n in self.STATE}

    def restore(self, state):
        for n, t in state.items():
            getattr(self, n).copy_(t)

    def rows(self, t, b):
        """[slots, Hkv, d] of sequence b."""
        return t[self.table[b].long()].flatten(0, 1)[: self.slots]


def test_steps_of_a_server():
    """Twenty steps: every slot holds the row of its position, sinks and the newest are there, and the
    attention is that of the rows held."""
    s = Server()
    T = len(s.pre.rows[0][0])
    assert T == 150
    for it in range(20):
        s.inputs()
        old = s.state()
        s.step()
        acc, lens, seq = (x.cpu().numpy() for x in (s.acc, s.lens, s.seq))
        assert (seq == old["seq"].cpu().numpy() + acc + 1).all()
        for b in range(s.B):
            for i in range(acc[b] + 1):
                s.history[b][int(old["seq"][b]) + i] = (s.k_new[b, i].clone(), s.v_new[b, i].clone())
            pos = s.pos[b].cpu().numpy()
            assert lens[b] == min(s.budget, int(s.before[b]))
            for h in range(s.Hkv):
                held = pos[h, : lens[b]].tolist()
                assert len(set(held)) == len(held)
                assert {p for p in range(seq[b]) if p < 2 or p >= seq[b] - 6} <= set(held)
                k, v = s.rows(s.k, b)[: lens[b], h], s.rows(s.v, b)[: lens[b], h]
                assert torch.equal(k, torch.stack([s.history[b][p][0][h] for p in held]))
                assert torch.equal(v, torch.stack([s.history[b][p][1][h] for p in held]))
        # The step's attention and weights against float64, from the caches it saw.
        n0 = old["lens"].cpu().numpy()
        n1 = n0 + s.L
        kb, vb = [], []
        for b in range(s.B):
            for old_t, new, out in ((old["k"], s.k_new, kb), (old["v"], s.v_new, vb)):
                out.append(np.concatenate([host(s.rows(old_t, b))[: n0[b]], host(new[b])]))
        ro, rl, mass, qk = plain.prefix_attention(host(s.q), kb, vb, n1, *s.pre.rows, [150, 120], None)
        top = max(float(np.abs(v).max()) for v in vb + s.pre.rows[1])
        ob, lb = plain.prefix_bounds("bf16", int(n1.max()) + T, ro, rl, mass, qk, s.d, top)
        assert (np.abs(host(s.o) - ro) <= ob).all() and (np.abs(host(s.lse) - rl) <= lb).all()
        lp = plain.token_logprobs(host(s.logits).reshape(-1, s.vocab), s.tokens.cpu().numpy().reshape(-1), 5)
        assert np.array_equal(s.top.cpu().numpy().reshape(-1, 5), lp[2])
        assert (s.top[:, :, 0][s.tokens >= 0] == s.tokens[s.tokens >= 0]).all()  # greedy: the most likely ones
        assert np.abs(host(s.lp).reshape(-1) - lp[0]).max() < 1e-4


def test_a_servers_step_as_a_graph():
    """Captured once and replayed over changing inputs, with eager steps between: bit for bit the eager
    step's; two such graphs share one workspace."""
    s = Server(seed=1)
    s.inputs()
    start = s.state()
    s.step()                                  # warm
    torch.cuda.synchronize()
    s.restore(start)
    graphs = []
    for _ in range(2):
        g, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side), torch.cuda.graph(g, stream=side):
            s.step()
        torch.cuda.current_stream().wait_stream(side)
        graphs.append(g)
    torch.cuda.synchronize()
    for rep in range(12):
        s.inputs()
        before = s.state()
        s.step()
        want = s.state()
        s.restore(before)
        s.ws.random_(0, 256)
        torch.cuda.synchronize()
        graphs[rep % 2].replay()
        torch.cuda.synchronize()
        for n, t in s.state().items():
            assert torch.equal(t.view(torch.uint8), want[n].view(torch.uint8)), (rep, n)


def test_another_stream_and_no_outputs_given():
    """Outputs and workspaces that the calls allocate belong to the call's stream."""
    s = Server(seed=2, B=4, L=2)
    s.inputs()
    s.step()
    side = torch.cuda.Stream()
    args = (s.q, s.k, s.v, s.kv_lens, s.pre.k, s.pre.v, s.pre.lens)
    kw = dict(page_table=s.table, prefix_page_table=s.pre.table, max_kv_len=s.slots)
    o, lse = md.md_prefix_attn(*args, **kw)
    lp = md.md_token_logprobs(s.logits, s.tokens, top_k=7)
    torch.cuda.synchronize()
    for _ in range(5):
        o2, lse2 = md.md_prefix_attn(*args, stream=side, **kw)
        lp2 = md.md_token_logprobs(s.logits, s.tokens, top_k=7, stream=side)
        torch.empty_like(o2).fill_(7)         # the current stream's own use of memory meanwhile
        side.synchronize()
        assert torch.equal(o, o2) and torch.equal(lse, lse2)
        assert all(torch.equal(a, b) for a, b in zip(lp, lp2))
    none, _ = md.md_prefix_attn(*args, return_lse=False, **kw)
    assert torch.equal(none, o) and md.md_prefix_attn(*args, return_lse=False, **kw)[1] is None
    assert md.md_token_logprobs(s.logits, with_entropy=False)[:2] == (None, None)


def test_calls_of_nothing():
    s = Server(seed=3)
    e, z = s.q[:0], s.lens[:0]
    o, lse = md.md_prefix_attn(e, s.k, s.v, z, s.pre.k, s.pre.v, s.pre.lens, page_table=s.table,
                               prefix_page_table=s.pre.table)
    assert o.shape == e.shape and lse.shape == e.shape[:3]
    md.md_kv_mass(e, s.k, z, lse, s.mass, s.pos, z, page_table=s.table)
    assert md.md_kv_evict(s.k, s.v, s.mass, s.pos, z, z, 8, page_table=s.table).shape == (0,)
    assert md.md_token_logprobs(s.logits[:0], s.tokens[:0], top_k=2)[2].shape == (0, s.L, 2)


@pytest.mark.parametrize("case", BAD_ON_GPU, ids=[f"{b[0]}-{b[2]}-{i}" for i, b in enumerate(BAD_ON_GPU)])
def test_malformed_tensors(case):
    name, over, match = case
    kw = {k: t.to(DEV) if isinstance(t, torch.Tensor) else t for k, t in {**host_call(name), **over}.items()}
    if "mass" in over:                        # keep its stride on the device
        kw["mass"] = torch.zeros((2, 2, 40), device=DEV)[:, :, ::2]
    with pytest.raises(ValueError, match=match):
        getattr(md, name)(**kw)


# ---- prefix attention: rows, pages and lengths that pick other kernels ----

@pytest.mark.parametrize("case", [
    # dt, Hq, Hkv, d, L, own lengths, prefix lengths, page, prefix page
    ("bf16", 4, 1, 128, 3, [3 + i for i in range(9)], [333], 1, 1),        # pages too small for shared tiles
    ("bf16", 4, 1, 128, 3, [3 + i for i in range(9)], [333], 2, 2),
    ("bf16", 4, 1, 64, 3, [3 + i for i in range(9)], [333], 4, 4),
    ("bf16", 4, 1, 64, 3, [3 + i for i in range(9)], [333], 8, 8),
    ("bf16", 4, 1, 128, 3, [3 + i for i in range(9)], [333], 16, 4),
    ("bf16", 4, 1, 128, 3, [3 + i for i in range(9)], [63], 16, 16),       # less than a tile, one, one more
    ("bf16", 4, 1, 128, 3, [3 + i for i in range(9)], [64], 16, 16),
    ("bf16", 4, 1, 128, 3, [3 + i for i in range(9)], [65], 16, 16),
    ("bf16", 4, 2, 128, 3, [3 + i for i in range(18)], [0, 2000], 64, 16), # one of two prefixes empty
    ("bf16", 4, 1, 64, 16, [16] * 5, [129], 0, 0),                         # 320 rows: two blocks
    ("bf16", 1, 1, 128, 1, [1] * 65, [4000], 0, 16),                       # 65 rows, one a sequence
    ("bf16", 4, 1, 64, 5, [5 + i for i in range(10)], [777], 0, 0),        # 200 rows: one block of 256
    ("bf16", 4, 1, 64, 5, [5 + i for i in range(10)], [777], 16, 16),
    ("bf16", 8, 1, 128, 4, [4 + i for i in range(30)], [500], 0, 0),       # 960: four
    ("bf16", 8, 1, 64, 3, [3] * 16, [31], 16, 16),                         # 384: three of 128
    ("f32", 4, 2, 64, 5, [2000, 5, 700], [3000], 16, 16),
    ("bf16", 4, 1, 128, 3, [3000, 2000, 1000, 4], [1], 16, 16),            # long own caches in parts
])
def test_prefix_kernels(case):
    check_prefix(*case)


@pytest.mark.parametrize("case", [
    # Groups of many rows over long prefixes: tiles that the waves of a workgroup share.
    ("bf16", 32, 8, 128, 1, [1 + i % 9 for i in range(48)], [16384 + 63], 0, 0),      # 192 rows, a tail of 63
    ("bf16", 32, 8, 128, 1, [1 + i % 9 for i in range(50)], [16384], 16, 4),          # whole tiles
    ("bf16", 32, 8, 64, 1, [1 + i % 9 for i in range(64)], [16384 + 65], 16, 8),      # 256 rows
    ("bf16", 32, 8, 64, 2, [2 + i % 9 for i in range(36)], [16384 + 1], 0, 0),        # 288: three of 128
    ("bf16", 32, 8, 128, 4, [4 + i % 9 for i in range(34)], [40, 16390], 16, 16),     # 272 and a short one beside
], ids=["192", "200", "256", "288", "272"])
def test_prefix_kernel_of_many_rows(case):
    check_prefix(*case)


def test_prefix_wide_rows_of_nan_and_infinity():
    """In tiles of many rows, too, a NaN query reaches its own row alone, and a NaN key every row."""
    gen = torch.Generator().manual_seed(7)
    own, pre = Cache(gen, [1] * 90, 1, 8, 128, "bf16"), Cache(gen, [17000], 17000, 8, 128, "bf16")
    q = rand(gen, (90, 1, 16, 128), "bf16")
    clean, l0 = md.md_prefix_attn(q, own.k, own.v, own.lens, pre.k, pre.v, pre.lens)
    bad = q.clone()
    bad[33, 0, 1, 5] = float("nan")
    o, lse = md.md_prefix_attn(bad, own.k, own.v, own.lens, pre.k, pre.v, pre.lens)
    assert o[33, 0, 1].isnan().all() and lse[33, 0, 1] == float("-inf")
    o[33, 0, 1], lse[33, 0, 1] = clean[33, 0, 1], l0[33, 0, 1]
    assert torch.equal(o, clean) and torch.equal(lse, l0)
    k = pre.k.clone()
    k[0, 333, 0, 0] = float("nan")
    o, lse = md.md_prefix_attn(q, own.k, own.v, own.lens, k, pre.v, pre.lens)
    assert o[:, :, :2].isnan().all() and (lse[:, :, :2] == float("-inf")).all()
    assert torch.equal(o[:, :, 2:], clean[:, :, 2:]) and torch.equal(lse[:, :, 2:], l0[:, :, 2:])
    huge = (q * 1e4).clamp(-3e4, 3e4)                                      # scores far past the exponential's range
    o, lse = md.md_prefix_attn(huge, own.k, own.v, own.lens, pre.k, pre.v, pre.lens)
    assert torch.isfinite(o.float()).all() and torch.isfinite(lse).all()


# ---- weights: long prompts in parts, odd groups ----

@pytest.mark.parametrize("case", [
    # dt, Hq, Hkv, d, L, lengths, accepted, page
    ("bf16", 8, 2, 128, 700, [700, 1500, 701], None, 16),     # a prompt behind cached tokens
    ("bf16", 6, 2, 64, 513, [513, 600], [400, 512], 0),       # groups that no tile holds whole
    ("bf16", 5, 1, 128, 300, [0, 300, 299, 1], None, 0),      # shorter than the prompt
    ("f32", 4, 2, 64, 257, [257], [0], 16),                   # one row counts
    ("f32", 7, 7, 128, 400, [400, 900], None, 0),
])
def test_mass_of_long_prompts(case):
    dt, Hq, Hkv, d, L, lens, acc, page = case
    gen = torch.Generator().manual_seed(L)
    c = Cache(gen, lens, max(max(lens), L), Hkv, d, dt, page)
    B, S = len(lens), max(max(lens), L) + 5
    q = rand(gen, (B, L, Hq, d), dt)
    lse = row_lse(host(q), c.rows[0], lens)
    mass, pos = torch.rand((B, Hkv, S), generator=gen), torch.full((B, Hkv, S), -7, dtype=I32)
    outs = []
    for fill in (0, 255):                      # whatever the workspace held, and the same bits each time
        m, x = mass.to(DEV), pos.to(DEV)
        a = dict(accepted=None if acc is None else ints(acc), max_kv_len=S - 5, page_table=c.table)
        ws = torch.full((1 << 22,), fill, dtype=torch.uint8, device=DEV)
        md.md_kv_mass(q, c.k, c.lens, torch.from_numpy(lse).to(DEV), m, x, ints([9 * b for b in range(B)]),
                      workspace=ws, **a)
        outs.append(m)
    assert torch.equal(outs[0], outs[1])
    want, wpos, err = plain.kv_mass(host(q), c.rows[0], lens, lse.astype(np.float64), mass.numpy().astype(np.float64),
                                    pos.numpy(), [9 * b for b in range(B)], acc)
    assert np.array_equal(x.cpu().numpy(), wpos)
    assert (np.abs(host(m) - want) <= err).all(), (np.abs(host(m) - want) - err).max()


def test_mass_of_rows_that_weigh_nothing():
    """Rows of lse -inf in a long prompt add nothing, whatever their queries hold."""
    gen = torch.Generator().manual_seed(12)
    L = 400
    c = Cache(gen, [L], L, 1, 64, "bf16")
    q = rand(gen, (1, L, 2, 64), "bf16")
    lse = row_lse(host(q), c.rows[0], [L])
    off = np.zeros((1, L, 2), dtype=bool)
    off[0, [3, 100, 101, 399]] = True
    off[0, 200:280, 1] = True
    lse[off] = -np.inf
    m, x = torch.zeros((1, 1, L), device=DEV), torch.zeros((1, 1, L), dtype=I32, device=DEV)
    md.md_kv_mass(q, c.k, c.lens, torch.from_numpy(lse).to(DEV), m, x, ints([0]))
    q2 = q.clone()
    q2[torch.from_numpy(off).to(DEV)] = float("nan")
    m2 = torch.zeros_like(m)
    md.md_kv_mass(q2, c.k, c.lens, torch.from_numpy(lse).to(DEV), m2, x, ints([0]))
    assert torch.equal(m, m2)
    want, _, err = plain.kv_mass(host(q), c.rows[0], [L], lse.astype(np.float64), np.zeros((1, 1, L)),
                                 np.zeros((1, 1, L)), [0])
    assert (np.abs(host(m) - want) <= err).all()


# ---- eviction and log probabilities at their edges ----

@pytest.mark.parametrize("slots,budget", [(30, 22), (30, 21), (9, 1), (600, 88), (600, 87), (1030, 517), (4097, 3585),
                                          (4097, 4096), (9000, 700)])
def test_evict_few_and_many(slots, budget):
    """Around the numbers of tokens evicted and moved at which the work is done in other ways."""
    lens = [slots, budget + 1, budget + 8, budget + 9, budget, budget - 1, slots + 40, -3]
    check_evict("bf16", 2, 64, lens, slots, budget, n_sink=min(3, budget // 3), recent=budget // 2, seed=slots)


def test_logprobs_of_a_large_vocabulary():
    """More logits a segment than a workgroup holds at once, with the largest ones in any of them."""
    V = (1 << 21) + 77
    gen = torch.Generator().manual_seed(1)
    x = rand(gen, (2, V), "bf16", 2.0)
    x[0, [5, 5000, 9000, V - 1]] = 20.0
    x[1, V // 2: V // 2 + 40] = 30.0
    check_logp(x, np.array([V - 1, 4096]), 32, chunks=4)


# ---- lengths up to the last ones, offsets past 32 bits ----

def test_the_longest_lengths():
    """2^31 - 65 shared tokens and 2^31 - 257 cached ones, one page of them again and again: token numbers
    of the tiles read ahead lie past 31 bits."""
    gen = torch.Generator().manual_seed(4)
    page, d, n = 1 << 20, 64, 2 ** 31 - 65
    k, v = (rand(gen, (1, page, 1, d), "bf16") for _ in "kv")
    k *= 0.1
    table = torch.zeros((1, 2048), dtype=I32, device=DEV)
    for rows in (4, 168):                    # a stream, and tiles that waves share
        q = rand(gen, (rows, 1, 1, d), "bf16")
        none = torch.zeros(rows, dtype=I32, device=DEV)
        own = torch.zeros((rows, 8, 1, d), dtype=torch.bfloat16, device=DEV)
        word = torch.zeros(1, dtype=I32, device=DEV)
        o, lse = md.md_prefix_attn(q, own, own, none, k, v, ints([n]), prefix_page_table=table, max_prefix_len=n,
                                   err_word=word)
        s = q[:, 0, 0].double() @ k[0, :, 0].double().T / 8.0
        assert int(word) == md.MD_ERRW_SHORT_LEN
        # 65 of 2^31 keys are missing: 2^-24 of the sum.  A lane adds 2^15 tiles' weights in fp32 (2^-9 at
        # most), and O two products of bf16 weights each (2^-8 and 2^-9 of mean |v| < 1).
        assert ((lse[:, 0, 0] - torch.logsumexp(s, 1) - np.log(2048.0)).abs() < 2 ** -8).all()
        want = torch.softmax(s, 1) @ v[0, :, 0].double()
        assert (o[:, 0, 0].double() - want).abs().max() < 2 ** -7
    n = 2 ** 31 - 257
    q = rand(gen, (1, 3, 2, d), "bf16")
    mass, pos = torch.zeros((1, 1, n), device=DEV), torch.zeros((1, 1, n), dtype=I32, device=DEV)
    lse = torch.full((1, 3, 2), 1.0, device=DEV)
    md.md_kv_mass(q, k, ints([n]), lse, mass, pos, ints([77]), page_table=table, max_kv_len=n)
    w = torch.exp(q[0].reshape(6, d).float() @ k[0, :, 0].float().T / 8.0 - 1.0).sum(0)
    for i in (0, 1000, 2046):
        assert torch.allclose(mass[0, 0, i * page:(i + 1) * page], w, rtol=1e-4)
    last = mass[0, 0, 2047 * page:]
    assert torch.allclose(last[:-2], w[: len(last) - 2], rtol=1e-4)     # the last three see fewer rows
    assert last[-1] < last[-2] or last[-1] < w[len(last) - 1]
    assert pos[0, 0, -3:].tolist() == [77, 78, 79] and not pos[0, 0, :-3].any()



def test_offsets_past_32_bits():
    """A page pool of more than 2^31 elements, used at its end; rows of logits as far apart."""
    gen = torch.Generator().manual_seed(3)
    Hkv, d, page, Hq = 8, 128, 16, 16
    pages = (1 << 31) // (Hkv * d * page) + 40
    small = Cache(gen, [40, 70, 33], 80, Hkv, d, "bf16", page)
    pre = Cache(gen, [200], 208, Hkv, d, "bf16", page)
    k, v = (torch.zeros((pages, page, Hkv, d), dtype=torch.bfloat16, device=DEV) for _ in "kv")
    n, m = small.k.shape[0], pre.k.shape[0]
    base = pages - n - m
    for t, a, b in ((k, small.k, pre.k), (v, small.v, pre.v)):
        t[base:base + n], t[base + n:] = a, b
    table, ptable = small.table + base, pre.table + base + n
    for L, seqs in ((2, 3), (11, 3)):
        q = rand(gen, (seqs, L, Hq, d), "bf16")
        a = md.md_prefix_attn(q, small.k, small.v, small.lens, pre.k, pre.v, pre.lens, page_table=small.table,
                              prefix_page_table=pre.table)
        b = md.md_prefix_attn(q, k, v, small.lens, k, v, pre.lens, page_table=table, prefix_page_table=ptable)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
        states = []
        for kk, tt in ((small.k, small.table), (k, table)):
            mass, pos = torch.zeros((3, Hkv, 80), device=DEV), torch.zeros((3, Hkv, 80), dtype=I32, device=DEV)
            md.md_kv_mass(q, kk, small.lens, a[1], mass, pos, ints([0, 5, 9]), page_table=tt)
            states.append((mass, pos))
        assert all(torch.equal(x, y) for x, y in zip(*states))
    # 192 rows of a prefix and KV head, 16400 tokens of it
    many, lens, rep = rand(gen, (3, 1, Hq, d), "bf16").repeat(32, 1, 1, 1), small.lens.repeat(32), 32
    pre.lens.fill_(16400)
    pre.table, ptable = (t[:, :12].repeat(1, 86)[:, :1025].contiguous() for t in (pre.table, ptable))
    a = md.md_prefix_attn(many, small.k, small.v, lens, pre.k, pre.v, pre.lens, page_table=small.table.repeat(rep, 1),
                          prefix_page_table=pre.table)
    b = md.md_prefix_attn(many, k, v, lens, k, v, pre.lens, page_table=table.repeat(rep, 1), prefix_page_table=ptable)
    assert torch.equal(a[0], b[0])
    for kk, vv, tt, (mass, pos) in ((small.k, small.v, small.table, states[0]), (k, v, table, states[1])):
        md.md_kv_evict(kk, vv, mass, pos, small.lens, ints([100] * 3), 30, page_table=tt)
    assert all(torch.equal(x, y) for x, y in zip(*states))
    for big, little in ((k, small.k), (v, small.v)):
        assert torch.equal(big[base:base + n].view(I32), little.view(I32))
        assert not big[:base].any()
    del k, v
    x = torch.zeros((1 << 31) + 9000, dtype=torch.bfloat16, device=DEV)
    rows = x.as_strided((2, 6000), ((1 << 31) + 1001, 1))
    rows.copy_(rand(gen, (2, 6000), "bf16", 2.0))
    check_logp(rows, np.array([5999, 17]), 9)
