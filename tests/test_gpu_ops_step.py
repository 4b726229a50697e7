"""One speculative step with sampled tokens, as a program strings the operators together: a
draft that reads a 4-bit copy of the cache, verification over the bf16 cache, acceptance by
probabilities and the commit.  Every operator's result is checked against float64 from its
inputs; then the whole step is captured in a graph and replayed."""
import numpy as np
import pytest
import torch

import paper_2408_11049_amd as md
import plain_ops as plain

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def host(t):
    return t.detach().to(torch.float64).cpu().numpy()


class Step:
    """A layer's attention with random projections between random embeddings and logits:
    enough of a model that each operator's output is the next one's input."""

    def __init__(self, lens, gamma, Hq=8, Hkv=2, d=64, vocab=1000, page=16, seed=0):
        g = torch.Generator().manual_seed(seed)

        def rand(*shape, scale=1.0):
            return (torch.randn(shape, generator=g) * scale).to(torch.bfloat16).to(DEV)
        self.B, self.gamma, self.Hq, self.Hkv, self.d, self.vocab = len(lens), gamma, Hq, Hkv, d, vocab
        B, L, n = self.B, gamma + 1, max(lens) + 2 * (gamma + 1)
        self.cap = -(-n // page) * page
        self.heads = Hq + 2 * Hkv
        self.embed = rand(vocab, self.heads * d)          # fused Q, K, V rows of a token
        self.out = rand(Hq * d, vocab, scale=0.2)
        self.qw, self.kw = 1 + rand(d, scale=0.1), 1 + rand(d, scale=0.1)
        self.inv = (10000.0 ** (-torch.arange(0, d, 2, dtype=torch.float64) / d)).float().to(DEV)
        cols = self.cap // page
        perm = torch.randperm(B * cols, generator=g).reshape(B, cols)
        self.table = perm.to(torch.int32).to(DEV)
        self.k = torch.zeros((B * cols, page, Hkv, d), dtype=torch.bfloat16, device=DEV)
        self.v = torch.zeros_like(self.k)
        self.small = md.kv4_empty(B, self.cap, Hkv, d, device=DEV)
        self.lens = torch.tensor(lens, dtype=torch.int32, device=DEV)
        # The prompt's rows, in both caches.
        zero = torch.zeros(B, dtype=torch.int32, device=DEV)
        prompt = torch.randint(0, vocab, (B, max(lens)), generator=g).to(DEV)
        q, kr, vr = self.project(prompt)
        _, ko, _ = self.norm(q, kr, zero, v_new=vr, k=self.k, v=self.v, page_table=self.table,
                             k_out=torch.empty(kr.shape, dtype=torch.bfloat16, device=DEV))
        md.md_kv4_append(self.small, ko, vr.contiguous(), zero)
        self.first = torch.randint(0, vocab, (B,), generator=g).to(DEV)
        self.noise = torch.rand((gamma, B, vocab), generator=g).clamp_min(1e-6).log().neg().to(DEV)
        self.u = torch.rand((B, L), generator=g).to(DEV)

    def project(self, tokens):
        rows = self.embed[tokens].view(*tokens.shape, self.heads, self.d)
        return rows.split([self.Hq, self.Hkv, self.Hkv], 2)  # views of one projection

    def norm(self, q, k_new, pos, **kw):
        return md.md_qk_norm_rope(q, k_new, pos, self.inv, q_weight=self.qw, k_weight=self.kw, **kw)

    def probs(self, o):
        B, L = o.shape[:2]
        return (o.reshape(B * L, -1).float() @ self.out.float()).softmax(-1).view(B, L, self.vocab)

    def run(self, seen=None):
        """seen: a list that takes (operator, inputs and results) for the checks."""
        seen = [] if seen is None else seen
        B, L = self.B, self.gamma + 1
        tok, drafts, qs, pos = self.first, [], [], self.lens
        for i in range(self.gamma):
            drafts.append(tok)
            q, k, v = self.project(tok[:, None])
            qn, kn, _ = self.norm(q, k, pos)
            pos = md.md_kv4_append(self.small, kn, v.contiguous(), pos)
            o, lse = md.md_kv4_verify_attn(qn, self.small, pos)
            seen.append(("draft", qn, pos, o, lse, [t.clone() for t in self.small]))
            pr = self.probs(o)[:, 0]
            qs.append(pr)
            tok = (pr / self.noise[i]).argmax(-1)  # a draw from pr
        drafts.append(tok)
        chain = torch.stack(drafts, 1)
        q, k, v = self.project(chain)
        kept = torch.empty(k.shape, dtype=torch.bfloat16, device=DEV)
        qn, _, kv_lens = self.norm(q, k, self.lens, v_new=v, k=self.k, v=self.v,
                                   page_table=self.table, k_out=kept)
        seen.append(("rows", q, k, self.lens.clone(), qn, kept))
        md.md_kv4_append(self.small, kept, v.contiguous(), self.lens)
        o, _ = md.md_verify_attn(qn, self.k, self.v, kv_lens, max_kv_len=self.cap,
                                 page_table=self.table)
        seen.append(("verify", qn, kv_lens, o))
        p, qp = self.probs(o), torch.stack(qs, 1)
        draft = chain[:, 1:].to(torch.int32).contiguous()
        acc, out = md.md_spec_accept(p, qp, draft, self.u)
        seen.append(("accept", p, qp, draft, acc, out))
        md.md_kv_commit(self.lens, acc, L)
        return acc, out, self.lens, o, qp, *self.small, self.k, self.v


def small_rows(cache):
    out = []
    for c, s in ((cache[0], cache[2]), (cache[1], cache[3])):
        out.append(plain.kv4_values(plain.unpack(c.cpu().numpy()), s.cpu().numpy().astype(np.int64)))
    return out


def test_every_operator_of_a_step():
    lens = [50, 7, 129, 1]
    st = Step(lens, 3)
    seen = []
    acc = st.run(seen)[0]
    for what, *x in seen:
        if what == "draft":
            q, pos, o, lse, cache = x
            k, v = small_rows(cache)
            n = host(pos).astype(int)
            ro, rl, mass, qk = plain.attention(host(q), [k[b, :n[b]] for b in range(st.B)],
                                               [v[b, :n[b]] for b in range(st.B)], n)
            top = max(float(np.abs(v[b, :n[b]]).max()) for b in range(st.B))
            ob, lb = plain.attention_bounds("bf16", int(n.max()), ro, rl, mass, qk, st.d, top)
            assert (np.abs(host(o) - ro) <= ob).all() and (np.abs(host(lse) - rl) <= lb).all()
        elif what == "rows":
            q, k, pos, qn, kn = x
            at = host(pos).astype(int)[:, None] + np.arange(q.shape[1])
            for raw, w, got in ((q, st.qw, qn), (k, st.kw, kn)):
                y, size = plain.norm_rope(host(raw), host(w), at, st.inv.double().cpu().numpy())
                assert (np.abs(host(got) - y) <= plain.norm_rope_bound("bf16", y, size, st.d)).all()
            # Both caches hold these rows now: the bf16 one as they are, the small one rounded.
            table, k4 = st.table.cpu().numpy(), small_rows(st.small)[0]
            want4 = plain.kv4_values(*plain.kv4_round(host(kn)))
            for b in range(st.B):
                for i, t in enumerate(at[b]):
                    assert torch.equal(st.k[table[b, t // 16], t % 16], kn[b, i])
                    assert np.array_equal(k4[b, t], want4[b, i])
        elif what == "verify":
            q, n, o = x
            rows = [[c[st.table[b].long()].reshape(-1, st.Hkv, st.d)[: int(n[b])] for c in (st.k, st.v)]
                    for b in range(st.B)]
            ro = plain.attention(host(q), [host(r[0]) for r in rows], [host(r[1]) for r in rows],
                                 host(n).astype(int))[0]
            assert np.abs(host(o) - ro).max() <= 2e-2
        else:
            p, qp, draft, a, out = x
            ra, rt = plain.spec_accept(host(p), host(qp), draft.cpu().numpy(), host(st.u))
            assert np.array_equal(a.cpu().numpy(), ra) and np.array_equal(out.cpu().numpy(), rt)
    assert st.lens.tolist() == [n + int(a) + 1 for n, a in zip(lens, acc)]


def test_drafts_of_the_same_rows_are_mostly_kept():
    """With draft and target over the same prompt, what is refused comes from the rounding of
    the cache alone: some drafts of many sequences are kept, and the output's tokens are the
    accepted drafts, then one more."""
    st = Step([40] * 32, 3, seed=5)
    acc, out = st.run()[:2]
    assert int(acc.sum()) > 0
    assert all(int((row >= 0).sum()) == int(a) + 1 for row, a in zip(out, acc))


def test_a_captured_step_replays():
    st = Step([300, 17, 1100], 2, Hq=8, Hkv=2, d=128, vocab=40000, seed=2)
    state = [st.lens, *st.small, st.k, st.v]
    before = [t.clone() for t in state]

    def restore():
        for t, s in zip(state, before):
            t.copy_(s)
    want = [t.clone() for t in st.run()]
    restore()
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        got = st.run()
    torch.cuda.current_stream().wait_stream(side)
    for rep in range(4):
        restore()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(got, want)):
            assert torch.equal(a, b), f"replay {rep}: result {i}"
        restore()  # the program's own eager step between two replays
        for a, b in zip(st.run(), want):
            assert torch.equal(a, b)
        torch.cuda.synchronize()
