"""Attention over a shared prefix on the GPU at its edges, against float64 formulas."""
import numpy as np
import pytest
import torch

import paper_2408_11049_amd as md
import plain_answers as plain
from prefix_wide_cases import CASES, Inputs
from test_gpu_answers import DEV, host, rand

pytestmark = pytest.mark.gpu


def test_error_word_without_prefix_tokens():
    """A bound of no shared tokens: the lengths are checked against it all the same, one prefix a group."""
    gen = torch.Generator().manual_seed(6)
    q, k = rand(gen, (4, 2, 4, 64), "bf16"), rand(gen, (4, 24, 1, 64), "bf16")
    empty = torch.empty((2, 0, 1, 64), dtype=torch.bfloat16, device=DEV)
    pages, table = rand(gen, (3, 16, 1, 64), "bf16"), torch.zeros((2, 1), dtype=torch.int32, device=DEV)

    def ints(*x):
        return torch.tensor(x, dtype=torch.int32, device=DEV)

    def bits(plens, lens=(20, 9, 2, 2)):
        words = []
        for pk, kw in ((empty, {}), (pages, dict(prefix_page_table=table))):
            word = torch.zeros(1, dtype=torch.int32, device=DEV)
            o, lse = md.md_prefix_attn(q, k, k, ints(*lens), pk, pk, ints(*plens), max_kv_len=20, max_prefix_len=0,
                                       err_word=word, **kw)
            n = [min(x, 20) for x in lens]
            rows, none = [host(k[b, :x]) for b, x in enumerate(n)], [np.zeros((0, 1, 64))] * 2
            ro, rl, mass, qk = plain.prefix_attention(host(q), rows, rows, n, none, none, [0, 0])
            ob, lb = plain.prefix_bounds("bf16", 20, ro, rl, mass, qk, 64, float(k.abs().max()))
            assert (np.abs(host(o) - ro) <= ob).all() and (np.abs(host(lse) - rl) <= lb).all()
            words.append(int(word))
        assert words[0] == words[1]
        return words[0]
    assert bits((0, 0)) == 0
    assert bits((0, 1)) == md.MD_ERRW_LONG_LEN and bits((7, 0)) == md.MD_ERRW_LONG_LEN
    assert bits((0, -1)) == md.MD_ERRW_SHORT_LEN
    assert bits((5, -5)) == md.MD_ERRW_LONG_LEN | md.MD_ERRW_SHORT_LEN
    assert bits((0, 0), (20, 9, 21, 2)) == md.MD_ERRW_LONG_LEN


def on_device(rows, cap, page, gen):
    """[n, cap, Hkv, d] or pages in random order and their table, of lists of [S, Hkv, d]; NaN where no token is."""
    Hkv, d = rows[0].shape[1:]
    cols = -(-cap // page) if page else 1
    toks = page or cap
    t = torch.full((len(rows) * cols, toks, Hkv, d), float("nan"), dtype=torch.bfloat16)
    table = torch.randperm(len(t), generator=gen).reshape(len(rows), cols) if page else torch.arange(len(t))[:, None]
    for b, r in enumerate(rows):
        for c in range(-(-len(r) // toks)):
            part = r[c * toks:(c + 1) * toks]
            t[table[b, c], :len(part)] = part
    return t.to(DEV), table.to(torch.int32).to(DEV) if page else None


@pytest.mark.parametrize("name", CASES)
def test_shared_tiles_of_short_prefixes(name):
    """Groups of many rows over prefixes that end anywhere in a tile, a block of one and a part, none and one of a
    tile a part among them; the same bits again."""
    c = Inputs(name)
    ints = {n: torch.tensor(x, dtype=torch.int32, device=DEV) for n, x in (("own", c.lens), ("pre", c.plens))}
    k, table = on_device(c.k, max(c.lens), c.page, torch.Generator().manual_seed(1))
    v, _ = on_device(c.v, max(c.lens), c.page, torch.Generator().manual_seed(1))
    pk, ptable = on_device(c.pk, c.bound, c.ppage, torch.Generator().manual_seed(2))
    pv, _ = on_device(c.pv, c.bound, c.ppage, torch.Generator().manual_seed(2))
    q = c.q.to(DEV)
    kw = dict(page_table=table, prefix_page_table=ptable, max_prefix_len=c.bound)
    o, lse = md.md_prefix_attn(q, k, v, ints["own"], pk, pv, ints["pre"], **kw)
    again = md.md_prefix_attn(q, k, v, ints["own"], pk, pv, ints["pre"], **kw)
    assert torch.equal(o, again[0]) and torch.equal(lse, again[1])
    for p in range(len(c.plens)):
        ro, rl, ob, lb = c.oracle(p)
        mine = slice(p * c.n, (p + 1) * c.n)
        eo, el = np.abs(host(o[mine]) - ro), np.abs(host(lse[mine]) - rl)
        assert (eo <= ob).all() and (el <= lb).all(), (c.plens[p], eo.max(), el.max())
