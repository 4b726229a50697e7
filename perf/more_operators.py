"""The operators of sampling several answers of one prompt in bounded caches, in their
plain form and as calls into this library.

Each case names its operation (`op`) and sizes:
  prefix  md_prefix_attn: attention of q_len tokens a sequence over a prefix that a group
          of sequences shares (read once for the group) and over the sequence's own cache;
  mass    md_kv_mass: the softmax weights that the queries give each cached token, from
          the attention's lse, added to what the token had;
  evict   md_kv_evict: a cache cut down to a budget of tokens, those of the least
          accumulated weight first, sinks and recent ones kept;
  logp    md_token_logprobs: log probabilities of given tokens, the entropy, and the most
          likely tokens.

Head shapes are those of this repository's workloads (32 or 64 query heads over 8 KV heads
of 128 channels, and small ones), as are contexts, batches, pages, the vocabulary and the
budget of 2049 tokens.
"""
import math
import random

import numpy as np
import torch

own = False                 # True: run() calls the library's kernels

DEV = "cuda:0"
VOCAB = 128256
BUDGET = 2049
MAX_PREFIX_FLOPS = 1.8e11   # of the largest prefix case
MAX_SCORES = 1 << 29        # (row, key) pairs of the largest mass case
MAX_CACHE_ELEMS = 1 << 28   # K elements of the largest mass, evict and prefix case
MAX_LOGITS = 64 * 5 * VOCAB
F32_SHARE = 8               # fp32 products cost several times those of bf16


def _md():
    import paper_2408_11049_amd as md
    return md


def _case(op, name, **kw):
    c = dict(op=op, name=name, B=1, Hq=32, Hkv=8, d=128, dtype="bf16", q_len=1, s_lo=1024,
             s_hi=1024, page=0, n_prefix=1, p_lo=0, p_hi=0, budget=0, n_sink=0, recent=0,
             kept=False, vocab=0, top_k=0)
    c.update(kw)
    return c


def listed():
    return [
        # A unit-test-sized fp32 model answering twice from one prompt: latency.
        _case("prefix", "prefix_tiny_f32", B=2, Hq=4, Hkv=1, d=64, dtype="f32", q_len=4, s_lo=40,
              s_hi=64, p_lo=256, p_hi=256),
        # One user's question answered eight times, token by token, paged.
        _case("prefix", "prefix_b8_8k", B=8, s_lo=90, s_hi=301, page=16, p_lo=8001, p_hi=8001),
        # A server whose whole batch carries one long system prompt.
        _case("prefix", "prefix_b64_32k", B=64, s_lo=64, s_hi=1024, page=16, p_lo=32768,
              p_hi=32768),
        # The same with five tokens a sequence to verify: the largest.
        _case("prefix", "prefix_b64_verify", B=64, q_len=5, s_lo=256, s_hi=2048, page=16,
              p_lo=32768, p_hi=32768),
        # Four prompts of other lengths, sixteen answers each, eight query heads a KV head.
        _case("prefix", "prefix_4x16", B=64, Hq=64, n_prefix=4, s_lo=100, s_hi=700, p_lo=2000,
              p_hi=16384),
        # One user's decoded token over a cache of a chat's length.
        _case("mass", "mass_b1_4k", q_len=1, s_lo=4001, s_hi=4001, page=16),
        # A batch's verified tokens over caches at their budget; a part of them is kept.
        _case("mass", "mass_step", B=64, q_len=5, s_lo=BUDGET, s_hi=BUDGET + 5, kept=True),
        # A whole prompt's own weights, as it enters the cache.
        _case("mass", "mass_prompt", q_len=4096, s_lo=4096, s_hi=4096),
        # Caches brought back to their budget after a step.
        _case("evict", "evict_step", B=64, s_lo=BUDGET - 1, s_hi=BUDGET + 5, budget=BUDGET,
              n_sink=16, recent=1024, q_len=5),
        # Prompts cut to the budget once.
        _case("evict", "evict_prompt", B=8, s_lo=16384, s_hi=32768, budget=BUDGET, n_sink=16,
              recent=1024, page=16),
        # One token of one user, an odd vocabulary.
        _case("logp", "logp_b1", vocab=50001, top_k=5),
        # The tokens of a batch's step with the repository's vocabulary.
        _case("logp", "logp_b64", B=64, q_len=5, vocab=VOCAB, top_k=20, dtype="f32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _flops(c):
    return 4.0 * c["B"] * c["q_len"] * c["Hq"] * c["d"] * (c["p_hi"] + c["s_hi"])


def draw(rng: random.Random):
    """One more case of the listed ranges: 1 to 128 sequences, 1 to 16 answers a prompt and
    more, prefixes to 65536 tokens, own caches of 1 to 8192, both head dims and dtypes,
    groups of 1 to 8 query heads, contiguous and paged, budgets of 64 to 4096."""
    op = rng.choice(["prefix", "prefix", "mass", "evict", "logp"])
    Hkv = rng.choice([1, 2, 3, 4, 8, 8, 8])
    G = rng.choice([1, 2, 4, 4, 7, 8])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    share = F32_SHARE if dtype == "f32" else 1
    c = dict(Hq=Hkv * G, Hkv=Hkv, d=rng.choice([64, 128, 128]), dtype=dtype,
             page=rng.choice([0, 16, 16, 64]))
    if op == "prefix":
        while True:
            c["n_prefix"], n = rng.choice([1, 1, 1, 2, 3, 8]), _log_int(rng, 1, 128)
            c["B"], c["q_len"] = c["n_prefix"] * n, rng.choice([1, 1, rng.randint(2, 8)])
            c["p_hi"], c["s_hi"] = _log_int(rng, 16, 65536), _log_int(rng, 8, 8192)
            cc = _case(op, "", **c)
            if (c["B"] <= 128 and _flops(cc) <= MAX_PREFIX_FLOPS / share and
                    c["B"] * c["s_hi"] * Hkv * c["d"] <= MAX_CACHE_ELEMS):
                break
        c["p_lo"] = c["p_hi"] if rng.random() < 0.4 else int(c["p_hi"] * rng.uniform(0.1, 1.0))
        c["s_lo"] = min(c["s_hi"], max(c["q_len"], int(c["s_hi"] * rng.uniform(0.1, 1.0))))
    elif op == "mass":
        prompt = rng.random() < 0.35
        while True:
            c["B"], c["s_hi"] = _log_int(rng, 1, 8 if prompt else 128), _log_int(rng, 64, 32768)
            c["q_len"] = c["s_hi"] if prompt else rng.choice([1, 1, rng.randint(2, 9)])
            if (c["B"] * c["Hq"] * c["q_len"] * c["s_hi"] <= MAX_SCORES // share and
                    c["B"] * c["s_hi"] * Hkv * c["d"] <= MAX_CACHE_ELEMS):
                break
        c["s_lo"] = c["s_hi"] if prompt or rng.random() < 0.5 else max(
            c["q_len"], int(c["s_hi"] * rng.uniform(0.3, 1.0)))
        c["kept"] = not prompt and rng.random() < 0.5
    elif op == "evict":
        step = rng.random() < 0.5
        while True:
            c["B"], c["budget"] = _log_int(rng, 1, 128), _log_int(rng, 64, 4096)
            c["s_hi"] = c["budget"] + (rng.randint(1, 8) if step else _log_int(rng, 16, 30000))
            if c["B"] * c["s_hi"] * Hkv * c["d"] <= MAX_CACHE_ELEMS // (2 if dtype == "f32" else 1):
                break
        c["s_lo"] = c["budget"] - 1 if step else rng.randint(c["budget"] // 2, c["s_hi"])
        c["n_sink"] = rng.choice([0, 4, 16])
        c["recent"] = rng.randint(0, c["budget"] - c["n_sink"])
    else:
        while True:
            c["B"], c["q_len"] = _log_int(rng, 1, 128), rng.randint(1, 9)
            c["vocab"] = _log_int(rng, 1000, VOCAB)
            if c["B"] * c["q_len"] * c["vocab"] <= MAX_LOGITS:
                break
        c["top_k"] = rng.choice([0, 1, 5, 20, rng.randint(2, 32)])
    c = _case(op, "", **c)
    del c["name"]
    return c


# ------------------------------------------------------------------ inputs --

def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _gen(seed, stream):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 128 + stream)
    return g


def _randn(shape, dtype, seed, stream):
    return torch.empty(shape, dtype=dtype, device=DEV).normal_(generator=_gen(seed, stream))


def _lens(lo, hi, n):
    """Lengths on the host (shape-defining: fixed per case, so that states of other seeds
    hold the same work); the first is the longest."""
    x = np.random.default_rng([lo, hi, n]).integers(lo, hi + 1, size=n)
    x[0] = hi
    return x.astype(np.int32)


def _cache(case, rows, cap, seed, stream):
    """K, V and page table (None: contiguous) of `rows` sequences of up to `cap` tokens;
    pages are placed in seeded random order."""
    Hkv, d, ps = case["Hkv"], case["d"], case["page"]
    cap = max(cap, 1)
    if not ps:
        blocks, toks, pt = rows, cap, None
    else:
        n = -(-cap // ps)
        blocks, toks = rows * n, ps
        pt = torch.randperm(blocks, generator=_gen(seed, stream), device=DEV)
        pt = pt.to(torch.int32).reshape(rows, n).contiguous()
    shape = (blocks, toks, Hkv, d)
    return (_randn(shape, _dtype(case), seed, stream + 1),
            _randn(shape, _dtype(case), seed, stream + 2), pt)


def _dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(DEV)


def prepare(case, seed):
    op, B, L, Hq, Hkv, d = (case[x] for x in ("op", "B", "q_len", "Hq", "Hkv", "d"))
    dt = _dtype(case)
    st = dict(case=case)
    if op == "logp":
        V = case["vocab"]
        st["logits"] = (torch.randn((B, L, V), generator=_gen(seed, 0), device=DEV) * 3).to(dt)
        # Sampled tokens: likely ones, drawn by the largest logit with noise.
        noise = torch.rand((B, L, V), generator=_gen(seed, 1), device=DEV).clamp_(min=1e-30)
        noise = noise.log_().neg_().log_().neg_()
        st["tokens"] = (st["logits"].float() + noise).argmax(2).to(torch.int32)
        if L > 1:                                   # a step's tokens end before its rows do
            n = np.random.default_rng([seed, B, L]).integers(1, L + 1, size=B)
            st["tokens"][torch.arange(L, device=DEV)[None] >= _dev(n)[:, None]] = -1
        return st
    lens = _lens(case["s_lo"], case["s_hi"], B)
    st["lens_np"], st["lens"] = lens, _dev(lens)
    cap = int(lens.max())
    st["k"], st["v"], st["pt"] = _cache(case, B, cap, seed, 10)
    if op == "prefix":
        plens = _lens(case["p_lo"], case["p_hi"], case["n_prefix"])
        st["plens_np"], st["plens"] = plens, _dev(plens)
        st["pk"], st["pv"], st["ppt"] = _cache(case, case["n_prefix"], int(plens.max()), seed, 20)
        st["q"] = _randn((B, L, Hq, d), dt, seed, 0)
        return st
    rng = np.random.default_rng(seed)
    if op == "mass":
        st["q"] = _randn((B, L, Hq, d), dt, seed, 0)
        st["lse"] = _row_lse(st)
        past = 1 + rng.integers(0, 1000, size=B).astype(np.int32)
        st["pos0"] = _dev(lens - L + (0 if L == case["s_hi"] else past))
        st["accepted"] = _dev(rng.integers(0, L, size=B).astype(np.int32)) if case["kept"] else None
        st["mass"] = torch.rand((B, Hkv, cap), generator=_gen(seed, 30), device=DEV)
        st["slot_pos"] = torch.randint(0, cap, (B, Hkv, cap), generator=_gen(seed, 31),
                                       device=DEV).to(torch.int32)
        return st
    # evict: a few tokens hold most of the weight, as trained attention does; slots hold the
    # tokens in any order, as earlier evictions leave them; a step's tokens come last.
    u = torch.rand((B, Hkv, cap), generator=_gen(seed, 30), device=DEV)
    st["mass"] = 0.05 / (u + 1e-3)
    seq = lens.astype(np.int64) + rng.integers(0, 3000, size=B)
    st["seq_lens"] = _dev(seq.astype(np.int32))
    order = torch.rand((B, Hkv, cap), generator=_gen(seed, 31), device=DEV)
    slot = torch.arange(cap, device=DEV)
    n, L = st["lens"].long()[:, None, None], min(L, case["s_lo"])
    order = torch.where(slot < n - L, order, 2.0 + slot.float() / cap)
    rank = order.argsort(2).argsort(2)              # distinct: the rank of each slot's token
    gap = (st["seq_lens"].long()[:, None, None] - n)
    st["slot_pos"] = torch.where(rank < n // 3, rank, rank + gap).to(torch.int32).contiguous()
    return st


# -------------------------------------------------------------- plain forms --

def _rows(t, pt):
    """Cache rows [blocks, toks, Hkv, x] in token order, [B, S, Hkv, x]."""
    return t if pt is None else t[pt.long()].flatten(1, 2)


def _grouped(q, Hkv):
    """q [B, L, Hq, d] -> fp32 [B, Hkv, L * G, d] (row i * G + g)."""
    B, L, Hq, d = q.shape
    return (q.float().reshape(B, L, Hkv, Hq // Hkv, d).permute(0, 2, 1, 3, 4)
            .reshape(B, Hkv, -1, d).contiguous())


def _seen(st, S):
    """[B, L * G, S]: whether row (i, g) sees own key j."""
    c = st["case"]
    L, G = c["q_len"], c["Hq"] // c["Hkv"]
    pos = st["lens"].long()[:, None] - L + torch.arange(L, device=DEV)
    return torch.arange(S, device=DEV) <= pos.repeat_interleave(G, 1)[..., None]


def _keys(t):
    """[B, S, Hkv, d] -> fp32 [B, Hkv, d, S]."""
    return t.float().permute(0, 2, 3, 1).contiguous()


def _row_lse(st):
    """lse [B, L, Hq] of the attention over the own cache, a few KV heads at a time."""
    c = st["case"]
    B, L, Hq, Hkv, d = (c[x] for x in ("B", "q_len", "Hq", "Hkv", "d"))
    q, S = _grouped(st["q"], Hkv), int(st["lens_np"].max())
    k, seen = _rows(st["k"], st["pt"])[:, :S], _seen(st, S)
    out = torch.empty((B, Hkv, q.shape[2]), device=DEV)
    for b in range(B):
        for h in range(Hkv):
            s = torch.matmul(q[b, h], k[b, :, h].float().t().contiguous()) / math.sqrt(d)
            out[b, h] = torch.logsumexp(s.masked_fill(~seen[b], -math.inf), 1)
    return out.reshape(B, Hkv, L, Hq // Hkv).permute(0, 2, 1, 3).reshape(B, L, Hq).contiguous()


def _plain_prefix(st):
    c = st["case"]
    B, L, Hq, d = st["q"].shape
    Hkv, P, S = c["Hkv"], c["n_prefix"], int(st["lens_np"].max())
    n, R = B // P, L * (Hq // Hkv)
    q = _grouped(st["q"], Hkv)
    so = torch.matmul(q, _keys(_rows(st["k"], st["pt"])[:, :S])) / math.sqrt(d)
    so = so.masked_fill(~_seen(st, S)[:, None], -math.inf)                    # [B, Hkv, R, S]
    qg = (q.reshape(P, n, Hkv, R, d).permute(0, 2, 1, 3, 4).reshape(P, Hkv, n * R, d)
          .contiguous())
    sp = torch.matmul(qg, _keys(_rows(st["pk"], st["ppt"]))) / math.sqrt(d)   # [P, Hkv, n R, T]
    T = sp.shape[3]
    sp = sp.masked_fill((torch.arange(T, device=DEV) >= st["plens"].long()[:, None])[:, None, None],
                        -math.inf)

    def per_seq(x):                                 # [P, Hkv, n R, y] -> [B, Hkv, R, y]
        return (x.reshape(P, Hkv, n, R, -1).permute(0, 2, 1, 3, 4).reshape(B, Hkv, R, -1))
    m = torch.maximum(so.amax(3, keepdim=True), per_seq(sp.amax(3, keepdim=True)))
    mg = m.reshape(P, n, Hkv, R, 1).permute(0, 2, 1, 3, 4).reshape(P, Hkv, n * R, 1)
    po = torch.exp(so - m)
    pp = torch.exp(sp - mg)
    l = po.sum(3, keepdim=True) + per_seq(pp.sum(3, keepdim=True))
    own_v = _rows(st["v"], st["pt"])[:, :S].float().permute(0, 2, 1, 3).contiguous()
    pre_v = _rows(st["pv"], st["ppt"]).float().permute(0, 2, 1, 3).contiguous()
    o = (torch.matmul(po, own_v) + per_seq(torch.matmul(pp, pre_v))) / l
    G = Hq // Hkv
    o = o.reshape(B, Hkv, L, G, d).permute(0, 2, 1, 3, 4).reshape(B, L, Hq, d)
    lse = (m + torch.log(l)).reshape(B, Hkv, L, G).permute(0, 2, 1, 3).reshape(B, L, Hq)
    return o.to(st["q"].dtype).contiguous(), lse.contiguous()


def _counted(st):
    """[B, L]: whether row i of sequence b counts."""
    L = st["case"]["q_len"]
    i = torch.arange(L, device=DEV)[None]
    if st["accepted"] is None:
        return (i >= 0).expand(st["q"].shape[0], L)
    return i <= st["accepted"].long()[:, None]


def _plain_mass(st):
    c = st["case"]
    B, L, Hq, Hkv, d = (c[x] for x in ("B", "q_len", "Hq", "Hkv", "d"))
    S, G = st["mass"].shape[2], Hq // Hkv
    lse = st["lse"].reshape(B, L, Hkv, G).permute(0, 2, 1, 3).reshape(B, Hkv, L * G, 1)
    s = torch.matmul(_grouped(st["q"], Hkv), _keys(_rows(st["k"], st["pt"])[:, :S])) / math.sqrt(d)
    w = torch.exp(s - lse)
    del s
    use = _seen(st, S) & _counted(st).repeat_interleave(G, 1)[..., None]
    w = w.masked_fill_(~use[:, None], 0.0).sum(2)                             # [B, Hkv, S]
    j = torch.arange(S, device=DEV)[None, None]
    n = st["lens"].long()[:, None, None]
    live, new = j < n, (j >= n - L) & (j < n)
    m, pos = st["mass"], st["slot_pos"]
    m.copy_(torch.where(live, torch.where(new, w, m + w), m))
    here = st["pos0"].long()[:, None, None] + j - (n - L)
    pos.copy_(torch.where(new, here, pos.long()).to(torch.int32))
    return {"mass": m, "slot_pos": pos}


def _plain_evict(st):
    c = st["case"]
    mass, pos = st["mass"], st["slot_pos"]
    B, Hkv, S = mass.shape
    K = c["budget"]
    n = st["lens"].long().clamp(max=S)
    j = torch.arange(S, device=DEV)[None, None]
    seq = st["seq_lens"].long()[:, None, None]
    held = (pos.long() < c["n_sink"]) | (pos.long() >= seq - c["recent"])
    key = torch.where(held, math.inf, mass.double())
    key = torch.where(j < n[:, None, None], key, math.nan)                    # sorted last
    rank = key.argsort(dim=2, stable=True).argsort(dim=2)
    out = (rank < (n - K)[:, None, None])                                     # evicted
    live = j < n[:, None, None]
    hole = out & (j < K)
    extra = live & ~out & (j >= K)
    # The x-th hole takes the x-th of the kept tokens behind the budget.
    hb, hh, hj = hole.nonzero(as_tuple=True)
    eb, eh, ej = extra.nonzero(as_tuple=True)

    def slots(b, t):
        if st["pt"] is None:
            return b, t
        ps = c["page"]
        return st["pt"].long()[b, t // ps], t % ps
    for t in (st["k"], st["v"]):
        src, dst = slots(eb, ej), slots(hb, hj)
        t[dst[0], dst[1], hh] = t[src[0], src[1], eh]
    for t in (mass, pos):
        t[hb, hh, hj] = t[eb, eh, ej]
    return {"k": st["k"], "v": st["v"], "mass": mass, "slot_pos": pos,
            "lens": st["lens"].clamp(max=K)}


def _plain_logp(st):
    x, tok = st["logits"].float(), st["tokens"].long()
    V, K = x.shape[2], st["case"]["top_k"]
    m = x.amax(2, keepdim=True)
    e = torch.exp(x - m)
    z = e.sum(2, keepdim=True)
    ent = torch.log(z) - (e * (x - m)).sum(2, keepdim=True) / z
    lse = m + torch.log(z)
    lp = x.gather(2, tok.clamp(min=0)[..., None]) - lse
    lp = torch.where(tok >= 0, lp[..., 0], torch.zeros_like(lp[..., 0]))
    ids, vals = [], []
    idx = torch.arange(V, device=DEV)
    left = x.clone() if K else x
    for _ in range(K):                              # ties: the lowest token
        top = left.amax(2, keepdim=True)
        i = torch.where(left == top, idx, V).amin(2, keepdim=True)
        ids.append(i)
        vals.append(top - lse)
        left.scatter_(2, i, -math.inf)
    shape = x.shape[:2] + (0,)
    ids = torch.cat(ids, 2) if K else torch.empty(shape, dtype=torch.int64, device=DEV)
    vals = torch.cat(vals, 2) if K else torch.empty(shape, device=DEV)
    return {"logprobs": lp, "entropy": ent[..., 0], "top": ids.to(torch.int32), "top_logprobs": vals}


# ---------------------------------------------------------------- one pass --

def _own(st):
    md, c = _md(), st["case"]
    op, pt = c["op"], st.get("pt")
    if op == "logp":
        lp, ent, ids, vals = md.md_token_logprobs(st["logits"], st["tokens"], top_k=c["top_k"])
        return {"logprobs": lp, "entropy": ent, "top": ids, "top_logprobs": vals}
    if op == "prefix":
        return md.md_prefix_attn(st["q"], st["k"], st["v"], st["lens"], st["pk"], st["pv"],
                                 st["plens"], max_kv_len=c["s_hi"], page_table=pt,
                                 max_prefix_len=c["p_hi"], prefix_page_table=st["ppt"])
    if op == "mass":
        md.md_kv_mass(st["q"], st["k"], st["lens"], st["lse"], st["mass"], st["slot_pos"],
                      st["pos0"], accepted=st["accepted"], max_kv_len=c["s_hi"], page_table=pt)
        return {"mass": st["mass"], "slot_pos": st["slot_pos"]}
    lens = md.md_kv_evict(st["k"], st["v"], st["mass"], st["slot_pos"], st["lens"],
                          st["seq_lens"], c["budget"], n_sink=c["n_sink"], recent=c["recent"],
                          page_table=pt)
    return {"k": st["k"], "v": st["v"], "mass": st["mass"], "slot_pos": st["slot_pos"],
            "lens": lens}


def run(st):
    if own:
        return _own(st)
    return {"prefix": _plain_prefix, "mass": _plain_mass, "evict": _plain_evict,
            "logp": _plain_logp}[st["case"]["op"]](st)


# -------------------------------------------------------------------- work --

def work(case):
    op, B, L, Hq, Hkv, d = (case[x] for x in ("op", "B", "q_len", "Hq", "Hkv", "d"))
    es = 4 if case["dtype"] == "f32" else 2
    if op == "logp":
        n, K = B * L, case["top_k"]
        return {"bytes": int(n * (case["vocab"] * es + 12 + 8 * K)), "flops": int(5 * n * case["vocab"])}
    lens = _lens(case["s_lo"], case["s_hi"], B).astype(np.float64)
    page = 4.0 / case["page"] if case["page"] else 0.0
    own_keys = lens.sum()
    if op == "prefix":
        pre = _lens(case["p_lo"], case["p_hi"], case["n_prefix"]).astype(np.float64).sum()
        return {"bytes": int((own_keys + pre) * (2 * Hkv * d * es + page) + B * L * Hq * (2 * d * es + 4)),
                "flops": int(4 * L * Hq * d * (own_keys + pre * (B // case["n_prefix"])))}
    if op == "mass":
        seen = (lens * L - L * (L - 1) / 2).sum()       # (row, key) pairs of one head
        return {"bytes": int(own_keys * (Hkv * (d * es + 8) + page) + B * L * (Hq * (d * es + 4) + 4 * Hkv)),
                "flops": int(2 * d * Hq * seen)}
    # evict: every token's weight and position read; the kept tokens behind the budget, of
    # those that weights put there about their share, move with both.
    K = case["budget"]
    over = np.maximum(lens - K, 0)
    share = np.minimum(K, over) * np.where(over > 0, K / np.maximum(lens, 1), 0)
    moved = float(np.where(over > 64, share, np.minimum(over, K)).sum())
    return {"bytes": int(Hkv * (8 * own_keys + moved * (4 * d * es + 16))), "flops": int(4 * Hkv * own_keys)}


# ------------------------------------------------------------------- exact --

def _exact_prefix(st):
    c = st["case"]
    B, L, Hq, d = st["q"].shape
    Hkv, n = c["Hkv"], B // c["n_prefix"]
    G = Hq // Hkv
    o = torch.zeros(st["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros(st["q"].shape[:3], dtype=torch.float64, device=DEV)

    def rows(t, pt, b, S):
        if pt is None:
            return t[b, :S].double().transpose(0, 1).contiguous()
        return t[pt[b].long()].flatten(0, 1)[:S].double().transpose(0, 1).contiguous()
    for b in range(B):
        S, T = int(st["lens_np"][b]), int(st["plens_np"][b // n])
        k = torch.cat([rows(st["pk"], st["ppt"], b // n, T), rows(st["k"], st["pt"], b, S)], 1)
        v = torch.cat([rows(st["pv"], st["ppt"], b // n, T), rows(st["v"], st["pt"], b, S)], 1)
        at = T + S - L + torch.arange(L, device=DEV)                  # query positions
        hide = torch.arange(T + S, device=DEV)[None] > at.repeat_interleave(G)[:, None]
        qb = st["q"][b].double().reshape(L, Hkv, G, d).transpose(0, 1).reshape(Hkv, L * G, d)
        for h in range(Hkv):
            s = torch.mm(qb[h], k[h].t().contiguous()) * d ** -0.5
            s[hide] = -math.inf
            z = torch.logsumexp(s, 1)
            oh = torch.mm(torch.exp(s - z[:, None]), v[h])
            o[b, :, h * G:(h + 1) * G] = oh.reshape(L, G, d)
            lse[b, :, h * G:(h + 1) * G] = z.reshape(L, G)
    return o, lse


def _exact_mass(st):
    c = st["case"]
    B, L, Hq, Hkv, d = (c[x] for x in ("B", "q_len", "Hq", "Hkv", "d"))
    G = Hq // Hkv
    mass = st["mass"].double()
    for b in range(B):
        S = int(st["lens_np"][b])
        keep = L if st["accepted"] is None else int(st["accepted"][b]) + 1
        kb = st["k"][b, :S] if st["pt"] is None else st["k"][st["pt"][b].long()].flatten(0, 1)[:S]
        mass[b, :, S - L:S] = 0.0
        for h in range(Hq):
            kh = kb[:, h // G].double()
            for i0 in range(0, keep, 1024):
                i1 = min(keep, i0 + 1024)
                s = torch.mm(st["q"][b, i0:i1, h].double(), kh.t().contiguous()) * d ** -0.5
                w = torch.exp(s - st["lse"][b, i0:i1, h].double()[:, None])
                mass[b, h // G, :S] += torch.tril(w, S - L + i0).sum(0)
    return {"mass": mass, "slot_pos": None}


def _exact_logp(st):
    x = st["logits"].double()
    p = torch.log_softmax(x, 2)
    tok = st["tokens"].long()
    lp = p.gather(2, tok.clamp(min=0)[..., None])[..., 0]
    K = st["case"]["top_k"]
    return {"logprobs": torch.where(tok < 0, 0.0, lp), "entropy": -(p.exp() * p).sum(2), "top": None,
            "top_logprobs": p.topk(K, 2).values if K else p[..., :0]}


def exact(case, seed):
    op = case["op"]
    if op == "evict":       # rows are moved as they are: nothing is computed
        return None
    st = prepare(case, seed)
    return {"prefix": _exact_prefix, "mass": _exact_mass, "logp": _exact_logp}[op](st)
