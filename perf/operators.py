"""The operators around a speculative step with a 4-bit draft cache and
sampling, in their plain form and as calls into this library.

Each case names its operation (`op`) and sizes:
  attn    md_kv4_verify_attn / md_kv4_draft_attn: attention of q_len tokens a
          sequence over a KV cache held in 4 bits (E2M1 values, one power-of-two
          scale for 32 channels), over the whole context or, with a window, over
          sinks and window;
  append  md_kv4_append, which rounds new K/V rows into that cache, and
          md_kv4_read, which gives the cache's values back;
  accept  md_spec_accept: drafted tokens kept or refused by the target's
          probabilities and given random numbers, and the token drawn after them;
  norm    md_qk_norm_rope: RMS norm of each query and key head and the rotation by
          position, with the K and V rows written into the cache.

Head shapes are those of this repository's workloads (32 or 64 query heads over
8 KV heads of 128 channels, and small ones), as are contexts, batches, pages,
and the vocabulary.  K has a few channels scaled up, as trained keys do.
Probabilities are softmaxes of normal logits, the draft's those of the target's
logits with noise; drafts are drawn from the draft's probabilities.
"""
import math
import random

import numpy as np
import torch

own = False                 # True: run() calls the library's kernels

DEV = "cuda:0"
VOCAB = 128256
MAX_CACHE_ELEMS = 1 << 31   # K elements of the largest attention case
MAX_ROW_ELEMS = 1 << 25     # K elements of the largest append case
MAX_PROB_ELEMS = 64 * 9 * VOCAB
MAX_NORM_ELEMS = 4 * 4096 * 48 * 128
F32_SHARE = 8               # fp32 queries cost several times the products


def _md():
    import paper_2408_11049_amd as md
    return md


def _case(op, name, **kw):
    c = dict(op=op, name=name, B=1, Hq=32, Hkv=8, d=128, dtype="bf16", q_len=1, s_lo=4096,
             s_hi=4096, page=0, n_sink=0, window=0, vocab=0, gamma=0, sampled=True, rot=0,
             interleaved=False, eps=1e-6)
    c.update(kw)
    if op == "norm" and not c["rot"]:
        c["rot"] = c["d"]
    return c


def listed():
    return [
        # The smallest attention: a unit-test-sized fp32 model, bound by latency and the host path.
        _case("attn", "attn_tiny_f32", B=2, Hq=4, Hkv=1, d=64, dtype="f32", q_len=4, s_lo=256,
              s_hi=256),
        # One interactive user drafting a token over a 4-bit copy of a short chat, paged.
        _case("attn", "attn_b1_4k", B=1, q_len=1, s_lo=4001, s_hi=4001, page=16),
        # A medium batch drafting one token at 8k, contiguous cache.
        _case("attn", "attn_b32_8k", B=32, q_len=1, s_lo=8192, s_hi=8192),
        # A continuous-batching server: ragged long contexts, five tokens each; the largest.
        _case("attn", "attn_b64_ragged", B=64, q_len=5, s_lo=16384, s_hi=32768, page=16),
        # A draft over sinks and window of the long 4-bit cache.
        _case("attn", "attn_b64_window", B=64, q_len=1, s_lo=32768, s_hi=32768, page=16,
              n_sink=16, window=1008),
        # Prompts entering the 4-bit cache.
        _case("append", "append_prompt", B=8, q_len=4096, s_lo=0, s_hi=15),
        # A step's verified tokens entering the pages of a large batch.
        _case("append", "append_step", B=64, q_len=5, s_lo=16, s_hi=59, page=16),
        # One user's step: latency.
        _case("accept", "accept_b1", B=1, gamma=4, vocab=32000, dtype="f32"),
        # A large batch with the repository's vocabulary.
        _case("accept", "accept_b64", B=64, gamma=4, vocab=VOCAB, dtype="f32"),
        # Greedy drafts (no draft probabilities), bf16 target probabilities, an odd vocabulary.
        _case("accept", "accept_b16_greedy", B=16, gamma=7, vocab=50001, sampled=False),
        # A step's tokens of a large batch on their way into the paged cache.
        _case("norm", "norm_step", B=64, q_len=5, s_lo=16, s_hi=59, page=16),
        # Prompts.
        _case("norm", "norm_prompt", B=4, q_len=4096, s_lo=0, s_hi=0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    """One more case of the listed ranges: batches of 1 to 128, contexts of 128 to
    131072 tokens, both head dims and dtypes, groups of 1 to 8 query heads,
    contiguous and paged, uniform and ragged."""
    op = rng.choice(["attn", "attn", "attn", "append", "accept", "norm"])
    Hkv = rng.choice([1, 2, 3, 4, 8, 8, 8])
    G = rng.choice([1, 2, 4, 4, 7, 8])
    d = rng.choice([64, 128, 128])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    page = rng.choice([0, 16, 16, 64])
    share = F32_SHARE if dtype == "f32" else 1
    c = dict(B=_log_int(rng, 1, 128), Hq=Hkv * G, Hkv=Hkv, d=d, dtype=dtype, page=page)
    if op == "attn":
        while True:
            c["B"], s_hi = _log_int(rng, 1, 128), _log_int(rng, 128, 131072)
            if c["B"] * s_hi * Hkv * d <= MAX_CACHE_ELEMS // share // 2:
                break
        c["s_hi"] = s_hi
        c["s_lo"] = s_hi if rng.random() < 0.4 else max(64, int(s_hi * rng.uniform(0.3, 1.0)))
        c["q_len"] = rng.choice([1, 1, rng.randint(2, 8)])
        if rng.random() < 0.25:
            c["n_sink"], c["window"] = rng.choice([0, 4, 16, 64]), _log_int(rng, 64, 2048)
    elif op in ("append", "norm"):
        limit = MAX_ROW_ELEMS if op == "append" else MAX_NORM_ELEMS
        heads = Hkv if op == "append" else Hkv * (G + 2)
        while True:
            c["B"], n = _log_int(rng, 1, 128), _log_int(rng, 1, 4096)
            if c["B"] * (n + 64) * heads * d <= limit // (2 if dtype == "f32" else 1):
                break
        c["q_len"], c["s_lo"], c["s_hi"] = n, 0, rng.randint(1, 60)
        if op == "norm":
            c["rot"] = rng.choice([d, d, d // 2])
            c["interleaved"] = rng.random() < 0.3
            c["eps"] = rng.choice([1e-6, 1e-5])
    else:
        while True:
            c["B"], c["gamma"] = _log_int(rng, 1, 128), rng.randint(1, 8)
            c["vocab"] = _log_int(rng, 1000, VOCAB)
            if c["B"] * (2 * c["gamma"] + 1) * c["vocab"] <= MAX_PROB_ELEMS:
                break
        c["sampled"] = rng.random() < 0.7
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


def _lens(case):
    """Lengths on the host (shape-defining: fixed per case, so that states of
    other seeds hold the same work)."""
    lo, hi, B = case["s_lo"], case["s_hi"], case["B"]
    n = np.random.default_rng([lo, hi, B]).integers(lo, hi + 1, size=B)
    n[0] = hi
    return n.astype(np.int32)


def _pages(case, cap, seed):
    """The number of blocks, tokens a block holds and the page table of a cache of
    `cap` tokens a sequence (pages placed in seeded random order)."""
    B, ps = case["B"], case["page"]
    if not ps:
        return B, cap, None
    n = -(-cap // ps)
    perm = torch.randperm(B * n, generator=_gen(seed, 4), device=DEV)
    return B * n, ps, perm.to(torch.int32).reshape(B, n).contiguous()


def _kv4_rows(case, seed, blocks, toks, stream):
    """Codes [blocks, Hkv, toks, d / 2] and scales [blocks, Hkv, toks, d / 32] of
    seeded rows, a slab of blocks at a time, as [blocks, toks, Hkv, x] views."""
    Hkv, d = case["Hkv"], case["d"]
    codes = torch.empty((blocks, Hkv, toks, d // 2), dtype=torch.uint8, device=DEV)
    scales = torch.empty((blocks, Hkv, toks, d // 32), dtype=torch.uint8, device=DEV)
    g = _gen(seed, stream)
    loud = torch.ones(d, device=DEV)
    if stream == 1:  # K: a few loud channels
        loud[np.random.default_rng(seed).permutation(d)[:4].tolist()] = 8.0
    slab = max(1, (1 << 28) // (Hkv * toks * d))
    for i in range(0, blocks, slab):
        x = torch.randn((min(slab, blocks - i), Hkv, toks, d), generator=g, device=DEV) * loud
        codes[i:i + slab], scales[i:i + slab] = _pack(x)
    return codes.permute(0, 2, 1, 3), scales.permute(0, 2, 1, 3)


def prepare(case, seed):
    op, B, L, Hq, Hkv, d = (case[x] for x in ("op", "B", "q_len", "Hq", "Hkv", "d"))
    dt = _dtype(case)
    st = dict(case=case)
    if op == "accept":
        g, V = case["gamma"], case["vocab"]
        t = torch.randn((B, g + 1, V), generator=_gen(seed, 0), device=DEV) * 2
        st["p"] = torch.softmax(t, 2).to(dt)
        q = torch.softmax(t[:, :g] + 0.7 * torch.randn((B, g, V), generator=_gen(seed, 1),
                                                       device=DEV), 2).to(dt)
        if case["sampled"]:
            st["q"] = q
            cdf = q.double().cumsum(2)
            u = torch.rand((B, g, 1), generator=_gen(seed, 2), device=DEV).double() * cdf[..., -1:]
            st["draft"] = (torch.searchsorted(cdf, u, right=True)[..., 0].clamp(max=V - 1)
                           .to(torch.int32).contiguous())
        else:
            st["q"], st["draft"] = None, q.argmax(2).to(torch.int32).contiguous()
        st["u"] = torch.rand((B, g + 1), generator=_gen(seed, 3), device=DEV)
        return st
    lens = _lens(case)
    st["lens_np"], st["lens"] = lens, torch.from_numpy(lens.copy()).to(DEV)
    cap = int(lens.max()) + (0 if op == "attn" else L)
    blocks, toks, st["pt"] = _pages(case, cap, seed)
    st["cap"] = toks if st["pt"] is None else st["pt"].shape[1] * toks
    if op == "norm":
        qkv = _randn((B, L, (Hq + 2 * Hkv) * d), dt, seed, 0)
        q, k, v = qkv.split([Hq * d, Hkv * d, Hkv * d], 2)
        st["q"], st["kn"], st["vn"] = (x.unflatten(2, (h, d)) for x, h in
                                       ((q, Hq), (k, Hkv), (v, Hkv)))
        st["qw"] = (1 + 0.1 * torch.randn(d, generator=_gen(seed, 5), device=DEV)).to(dt)
        st["kw"] = (1 + 0.1 * torch.randn(d, generator=_gen(seed, 6), device=DEV)).to(dt)
        r = case["rot"]
        st["inv"] = (500000.0 ** (-torch.arange(0, r, 2, dtype=torch.float64) / r)).float().to(DEV)
        st["k"] = _randn((blocks, toks, Hkv, d), dt, seed, 1)
        st["v"] = _randn((blocks, toks, Hkv, d), dt, seed, 2)
        return st
    st["k4"], st["ks"] = _kv4_rows(case, seed, blocks, toks, 1)
    st["v4"], st["vs"] = _kv4_rows(case, seed, blocks, toks, 2)
    if op == "attn":
        st["q"] = _randn((B, L, Hq, d), dt, seed, 0)
    else:
        st["kn"] = _randn((B, L, Hkv, d), dt, seed, 7)
        st["kn"][..., np.random.default_rng(seed).permutation(d)[:4].tolist()] *= 8
        st["vn"] = _randn((B, L, Hkv, d), dt, seed, 8)
        st["zero"] = torch.zeros_like(st["lens"])
    return st


# -------------------------------------------------------------- plain forms --

def _pack(x):
    """x [..., d] fp32 -> codes [..., d / 2] and scales [..., d / 32], uint8."""
    blk = x.unflatten(-1, (-1, 32))
    a = blk.abs().amax(-1, keepdim=True)
    m, ex = torch.frexp(a)                       # a = m 2^ex, m in [0.5, 1)
    e = ex - 3 + (m >= 0.875).to(ex.dtype)
    e = torch.where(a == 0, torch.full_like(e, -125), e.clamp(-125, 125))
    y = torch.ldexp(blk.abs(), -e)               # exact: a power of two
    # The number of steps passed; a tie goes to the even code.
    code = torch.zeros_like(y, dtype=torch.uint8)
    code += y > 0.25
    code += y >= 0.75
    code += y > 1.25
    code += y >= 1.75
    code += y > 2.5
    code += y >= 3.5
    code += y > 5.0
    code += torch.signbit(blk).to(torch.uint8) * 8
    bad = ~torch.isfinite(blk).all(-1, keepdim=True)
    code = torch.where(bad, torch.zeros_like(code), code).flatten(-2)
    scale = torch.where(bad, torch.full_like(e, 255), e + 127)[..., 0].to(torch.uint8)
    return code[..., 0::2] | (code[..., 1::2] << 4), scale


_E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0]


def _unpack(codes, scales):
    """The values, fp32 [..., d]."""
    pairs = torch.tensor([[_E2M1[i & 15], _E2M1[i >> 4]] for i in range(256)], device=codes.device)
    s = torch.where(scales == 255, torch.full((), math.nan, device=scales.device),
                    (scales.to(torch.int32) << 23).view(torch.float32))
    x = pairs[codes.to(torch.int32)].flatten(-2).unflatten(-1, (-1, 32))
    return (x * s[..., None]).flatten(-2)


def _logical(t, pt):
    """Cache rows [blocks, toks, Hkv, x] in token order, [B, S, Hkv, x]."""
    return t if pt is None else t[pt.long()].flatten(1, 2)


def _slots(st, pos):
    """Block and token of the positions [B, n]: [B, n] each."""
    if st["pt"] is None:
        return torch.arange(pos.shape[0], device=DEV)[:, None].expand_as(pos), pos
    ps = st["case"]["page"]
    return st["pt"].long().gather(1, pos // ps), pos % ps


def _new_slots(st, n):
    """Block and token of the positions lens[b] + i, i < n."""
    return _slots(st, st["lens"].long()[:, None] + torch.arange(n, device=DEV))


def _plain_attn(st):
    c = st["case"]
    q, lens = st["q"].float(), st["lens"].long()
    B, L, Hq, d = q.shape
    Hkv, S = c["Hkv"], int(st["lens_np"].max())
    G = Hq // Hkv
    if c["window"]:          # sinks, then the windows of the L queries
        sinks = torch.arange(c["n_sink"], device=DEV).expand(B, -1)
        tail = lens[:, None] - L - c["window"] + 1 + torch.arange(c["window"] + L - 1, device=DEV)
        j = torch.cat([sinks, torch.where(tail < c["n_sink"], -1, tail)], 1)
        at = _slots(st, j.clamp(min=0))

        def rows(codes, scales):
            return _unpack(codes[at], scales[at])
    else:
        j = torch.arange(S, device=DEV)[None]

        def rows(codes, scales):
            return _logical(_unpack(codes, scales), st["pt"])[:, :S]
    j = j[..., None]
    k = rows(st["k4"], st["ks"]).permute(0, 2, 1, 3).contiguous()             # [B, Hkv, S, d]
    qt = q.reshape(B, L, Hkv, G, d).permute(0, 2, 4, 1, 3).reshape(B, Hkv, d, L * G)
    s = torch.matmul(k, qt) / math.sqrt(d)                                    # [B, Hkv, S, R]
    del k
    pos = (lens[:, None] - L + torch.arange(L, device=DEV)).repeat_interleave(G, 1)[:, None]
    vis = (j >= 0) & (j <= pos)                                               # [B, S, R]
    if c["window"]:
        vis = vis & ((j < c["n_sink"]) | (j > pos - c["window"]))
    s = s.masked_fill(~vis[:, None], -math.inf)
    m = s.amax(2, keepdim=True)
    p = torch.exp(s - m)
    l = p.sum(2, keepdim=True)
    v = rows(st["v4"], st["vs"]).permute(0, 2, 1, 3).contiguous()
    o = torch.matmul(p.transpose(2, 3).contiguous(), v) / l.transpose(2, 3)
    o = o.reshape(B, Hkv, L, G, d).permute(0, 2, 1, 3, 4).reshape(B, L, Hq, d)
    lse = (m + torch.log(l)).reshape(B, Hkv, L, G).permute(0, 2, 1, 3).reshape(B, L, Hq)
    return o.to(st["q"].dtype), lse.contiguous()


def _plain_append(st):
    n = st["kn"].shape[1]
    at = _new_slots(st, n)
    out = {}
    for x, new, codes, scales in (("k", "kn", "k4", "ks"), ("v", "vn", "v4", "vs")):
        c, s = _pack(st[new].float())
        st[codes][at] = c
        st[scales][at] = s
        out[x] = _logical(_unpack(st[codes], st[scales]), st["pt"]).to(torch.bfloat16).contiguous()
    out["lens"] = st["lens"] + n
    return out


def _plain_accept(st):
    p, q, draft, u = st["p"], st["q"], st["draft"].long(), st["u"]
    B, g = draft.shape
    V = p.shape[2]
    pd = p[:, :g].gather(2, draft[..., None])[..., 0].double()
    qd = torch.ones_like(pd) if q is None else q.gather(2, draft[..., None])[..., 0].double()
    a = (u[:, :g].double() * qd < pd).to(torch.int64).cumprod(1).sum(1)
    b = torch.arange(B, device=DEV)
    row = p[b, a].double()
    at = a.clamp(max=g - 1)
    if q is None:
        less = (torch.arange(V, device=DEV) == draft[b, at][:, None]).double()
    else:
        less = q[b, at].double()
    r = torch.where((a < g)[:, None], (row - less).clamp(min=0), row)
    r = torch.where(r.sum(1, keepdim=True) > 0, r, row)
    cdf = r.cumsum(1)
    tok = (cdf <= u[:, g:].double() * cdf[:, -1:]).sum(1)
    i = torch.arange(g + 1, device=DEV)
    drafts = torch.cat([draft, draft[:, :1]], 1)
    out = torch.where(i < a[:, None], drafts, torch.where(i == a[:, None], tok[:, None], -1))
    return a.to(torch.int32), out.to(torch.int32)


def _plain_norm(st):
    c = st["case"]
    L, r = c["q_len"], c["rot"]
    pos = st["lens"].double()[:, None] + torch.arange(L, device=DEV)
    ang = pos[..., None] * st["inv"].double()                     # far positions: 64 bits
    cos, sin = torch.cos(ang).float()[:, :, None], torch.sin(ang).float()[:, :, None]

    def rotated(x, w):
        x = x.float()
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + c["eps"]) * w.float()
        a, rest = x[..., :r], x[..., r:]
        if c["interleaved"]:
            x1, x2 = a[..., 0::2], a[..., 1::2]
            a = torch.stack([x1 * cos - x2 * sin, x2 * cos + x1 * sin], -1).flatten(-2)
        else:
            x1, x2 = a[..., : r // 2], a[..., r // 2:]
            a = torch.cat([x1 * cos - x2 * sin, x2 * cos + x1 * sin], -1)
        return torch.cat([a, rest], -1).to(st["q"].dtype)

    at = _new_slots(st, L)
    st["k"][at] = rotated(st["kn"], st["kw"])
    st["v"][at] = st["vn"]
    return {"q": rotated(st["q"], st["qw"]), "k": st["k"], "v": st["v"], "lens": st["lens"] + L}


# ---------------------------------------------------------------- one pass --

def _own(st):
    md, c = _md(), st["case"]
    op, pt = c["op"], st.get("pt")
    if op == "accept":
        return md.md_spec_accept(st["p"], st["q"], st["draft"], st["u"])
    if op == "norm":
        q, _, lens = md.md_qk_norm_rope(st["q"], st["kn"], st["lens"], st["inv"],
                                        q_weight=st["qw"], k_weight=st["kw"], eps=c["eps"],
                                        interleaved=c["interleaved"], v_new=st["vn"],
                                        k=st["k"], v=st["v"], page_table=pt)
        return {"q": q, "k": st["k"], "v": st["v"], "lens": lens}
    cache = md.Kv4Cache(st["k4"], st["v4"], st["ks"], st["vs"])
    if op == "append":
        lens = md.md_kv4_append(cache, st["kn"], st["vn"], st["lens"], page_table=pt)
        k, v = md.md_kv4_read(cache, st["zero"], st["cap"], page_table=pt)
        return {"k": k, "v": v, "lens": lens}
    kw = dict(max_kv_len=int(st["lens_np"].max()), page_table=pt)
    if c["window"]:
        return md.md_kv4_draft_attn(st["q"], cache, st["lens"], c["n_sink"], c["window"], **kw)
    return md.md_kv4_verify_attn(st["q"], cache, st["lens"], **kw)


def run(st):
    if own:
        return _own(st)
    return {"attn": _plain_attn, "append": _plain_append, "accept": _plain_accept,
            "norm": _plain_norm}[st["case"]["op"]](st)


# -------------------------------------------------------------------- work --

def work(case):
    op, B, L, Hq, Hkv, d = (case[x] for x in ("op", "B", "q_len", "Hq", "Hkv", "d"))
    es = 4 if case["dtype"] == "f32" else 2
    row4 = Hkv * (d // 2 + d // 32)                # one token's K (or V) in 4 bits
    if op == "accept":                             # one row of p, and of q where it has one
        V = case["vocab"]
        return {"bytes": int(B * V * es * (2 if case["sampled"] else 1)), "flops": int(3 * B * V)}
    lens = _lens(case).astype(np.float64)
    pages = 4.0 / case["page"] if case["page"] else 0.0
    if op == "attn":
        vis = lens
        if case["window"]:
            vis = np.minimum(lens, case["n_sink"] + case["window"] + L - 1)
        n = float(vis.sum())
        return {"bytes": int(n * (2 * row4 + pages) + B * L * Hq * (2 * d * es + 4)),
                "flops": int(4 * n * L * Hq * d)}
    if op == "append":                             # rows in, codes out, the whole cache's values back
        cap = (int(lens.max()) + L) if not case["page"] else -(-(int(lens.max()) + L) // case["page"]) * case["page"]
        n = B * L
        return {"bytes": int(2 * n * (Hkv * d * es + row4) + 2 * B * cap * (row4 + 2 * Hkv * d)),
                "flops": int(2 * (4 * n + B * cap) * Hkv * d)}
    n = B * L
    return {"bytes": int(2 * n * (Hq + 2 * Hkv) * d * es), "flops": int(8 * n * (Hq + Hkv) * d)}


# ------------------------------------------------------------------- exact --

def _values64(codes, scales):
    """sign * (1 + m / 2) * 2^(x - 1) (m / 2 where x = 0), times 2^(scale - 127): in 64 bits."""
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    x, m = ((c >> 1) & 3).double(), (c & 1).double()
    mag = torch.where(x == 0, m / 2, (1 + m / 2) * torch.exp2(x - 1))
    mag = torch.where(c >= 8, -mag, mag).unflatten(-1, (-1, 32))
    s = torch.exp2(scales.double() - 127)
    return (mag * torch.where(scales == 255, math.nan, s)[..., None]).flatten(-2)


def _rounded64(x):
    """The values that rows x are held as: the nearest level, ties to the even one."""
    x = x.double().unflatten(-1, (-1, 32))
    a = x.abs().amax(-1, keepdim=True)
    e = torch.floor(torch.log2(torch.where(a == 0, 1.0, a) * (8.0 / 7.0))) - 2
    # The logarithm can be off by an ulp where a is next to 7/8 of a power of two.
    e = torch.where(a * 8 / 7 >= torch.exp2(e + 3), e + 1, torch.where(a * 8 / 7 < torch.exp2(e + 2), e - 1, e))
    step = torch.exp2(e.clamp(-125, 125))
    y = x / step
    mag = y.abs().clamp(max=6.0)
    grid = torch.where(mag < 2, 0.5, torch.where(mag < 4, 1.0, 2.0))
    return (torch.copysign(torch.round(mag / grid) * grid, y) * step).flatten(-2)


def _exact_attn(st):
    c, q, lens = st["case"], st["q"], st["lens_np"]
    B, L, Hq, d = q.shape
    Hkv, ps = c["Hkv"], c["page"]
    G = Hq // Hkv
    o = torch.zeros(q.shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros(q.shape[:3], dtype=torch.float64, device=DEV)
    for b in range(B):
        S = int(lens[b])

        def rows(codes, scales):
            if st["pt"] is None:
                x = _values64(codes[b, :S], scales[b, :S])
            else:
                ids = st["pt"][b, : -(-S // ps)].long()
                x = _values64(codes[ids], scales[ids]).flatten(0, 1)[:S]
            return x.transpose(0, 1).contiguous()                             # [Hkv, S, d]

        qb = q[b].double().reshape(L, Hkv, G, d).permute(1, 0, 2, 3).reshape(Hkv, L * G, d)
        s = torch.matmul(rows(st["k4"], st["ks"]), qb.transpose(1, 2).contiguous())
        s = s.transpose(1, 2) / math.sqrt(d)                                  # [Hkv, R, S]
        j = torch.arange(S, device=DEV)[None]
        pos = (S - L + torch.arange(L, device=DEV)).repeat_interleave(G)[:, None]
        seen = (j <= pos) & ((j >= pos - c["window"] + 1) | (j < c["n_sink"]) if c["window"] else True)
        s = s.masked_fill(~seen[None], -math.inf)
        lb = torch.logsumexp(s, 2)
        ob = torch.matmul(torch.exp(s - lb[..., None]), rows(st["v4"], st["vs"]))
        o[b] = ob.reshape(Hkv, L, G, d).permute(1, 0, 2, 3).reshape(L, Hq, d)
        lse[b] = lb.reshape(Hkv, L, G).permute(1, 0, 2).reshape(L, Hq)
    return o, lse


def _exact_rows(st, caches, rows):
    """Caches (64-bit, [blocks, toks, Hkv, d]) with rows[i] written at positions lens[b] + i."""
    pt = None if st["pt"] is None else st["pt"].cpu().numpy()
    for cache, new in zip(caches, rows):
        for b, n0 in enumerate(st["lens_np"].tolist()):
            if pt is None:
                cache[b, n0:n0 + new.shape[1]] = new[b]
            else:
                ps = cache.shape[1]
                p = np.arange(n0, n0 + new.shape[1])
                cache[pt[b, p // ps].tolist(), (p % ps).tolist()] = new[b]
    return caches


def _exact_norm(st):
    c = st["case"]
    L, r = c["q_len"], c["rot"]
    pos = torch.from_numpy(st["lens_np"].astype(np.float64)[:, None] + np.arange(L)).to(DEV)
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV),
                       pos[..., None] * st["inv"].double())[:, :, None]

    def rotated(x, w):
        x = x.double()
        x = x / torch.sqrt((x ** 2).mean(-1, keepdim=True) + c["eps"]) * w.double()
        h = x[..., :r].unflatten(-1, (-1, 2) if c["interleaved"] else (2, -1))
        h = h if c["interleaved"] else h.transpose(-1, -2)
        z = torch.view_as_real(torch.view_as_complex(h.contiguous()) * turn)
        z = z if c["interleaved"] else z.transpose(-1, -2)
        return torch.cat([z.flatten(-2), x[..., r:]], -1)

    k, v = _exact_rows(st, [st["k"].double(), st["v"].double()],
                       [rotated(st["kn"], st["kw"]), st["vn"].double()])
    return {"q": rotated(st["q"], st["qw"]), "k": k, "v": v, "lens": None}


def _exact_accept(st):
    p, draft, u = (st[x].double().cpu().numpy() for x in ("p", "draft", "u"))
    q = None if st["q"] is None else st["q"].double().cpu().numpy()
    B, g = draft.shape
    kept, tokens = np.zeros(B, np.int32), np.full((B, g + 1), -1, np.int32)
    for b in range(B):
        d = draft[b].astype(np.int64)
        a = 0
        while a < g and u[b, a] * (1.0 if q is None else q[b, a, d[a]]) < p[b, a, d[a]]:
            a += 1
        r = p[b, a].copy()
        if a < g and q is None:
            r[d[a]] = max(r[d[a]] - 1.0, 0.0)
        elif a < g:
            r = np.maximum(r - q[b, a], 0.0)
        cdf = np.cumsum(r if r.sum() > 0 else p[b, a])
        kept[b], tokens[b, :a] = a, d[:a]
        tokens[b, a] = np.searchsorted(cdf, u[b, g] * cdf[-1], side="right")
    return kept, tokens


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "attn":
        return _exact_attn(st)
    if case["op"] == "accept":
        return _exact_accept(st)
    if case["op"] == "norm":
        return _exact_norm(st)
    k, v = _exact_rows(st, [_values64(st["k4"], st["ks"]), _values64(st["v4"], st["vs"])],
                       [_rounded64(st["kn"]), _rounded64(st["vn"])])
    order = (lambda t: t) if st["pt"] is None else (lambda t: t[st["pt"].long()].flatten(1, 2))
    return {"k": order(k), "v": order(v), "lens": None}
