"""Token log probabilities on the GPU at their edges: waves without logits, logits far from zero."""
import numpy as np
import pytest
import torch

import paper_2408_11049_amd as md
import plain_answers as plain
from test_gpu_answers import DEV, DT, check_logp, host, rand

pytestmark = pytest.mark.gpu

@pytest.mark.parametrize("rows,vocab,top_k", [
    (700, 40, 32), (700, 1000, 20), (700, 1025, 20), (300, 2049, 32), (300, 4096 + 60, 5), (300, 16384 + 300, 20)])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_logprobs_of_waves_without_logits(rows, vocab, top_k, dt):
    """Some of a workgroup's four waves have no logits, or one vector of them, and are done while the others read
    the bound on the top tokens: the same tokens, and the same bits call after call."""
    gen = torch.Generator().manual_seed(vocab)
    x = rand(gen, (rows, vocab), dt, 3.0)
    tok = torch.randint(-1, vocab, (rows,), generator=gen).numpy()
    check_logp(x, tok, top_k)
    t = torch.from_numpy(tok.astype(np.int32)).to(DEV)
    first = md.md_token_logprobs(x, t, top_k=top_k)
    for _ in range(20):
        again = md.md_token_logprobs(x, t, top_k=top_k)
        assert all(torch.equal(a, b) for a, b in zip(first, again))


LOW = float(torch.finfo(torch.float32).min)


def far_logprobs(x, tokens, top_k):
    """x [rows, V] float64: the log probabilities of tokens, the top_k tokens with theirs, and ln z, with (x - max) and
    ln z apart (at 1e30 their sum loses ln z in float64 too)."""
    m = x.max(1, keepdims=True)
    with np.errstate(invalid="ignore", divide="ignore"):
        d = np.where(x == -np.inf, -np.inf, x - m)
        lz = np.log(np.exp(d).sum(1, keepdims=True))
    at = np.arange(len(x))[:, None]
    top = np.argsort(-x, axis=1, kind="stable")[:, :top_k]

    def of(i):
        return np.where(x[at, i] == -np.inf, -np.inf, d[at, i] - np.where(np.isfinite(lz), lz, 0))
    return of(tokens[:, None])[:, 0], top, of(top), np.where(np.isfinite(lz), lz, 0)[:, 0]


@pytest.mark.parametrize("vocab,repeat", [(3000, 1), (9000, 1), (9000, 60), (40000, 60)])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_logprobs_of_logits_far_from_zero(vocab, repeat, dt):
    """A log probability is (x - max) - ln z: off by what these two and their difference are rounded by, wherever
    the logits lie.  logprob_bound with ln z in the place of lse's size says that much: the sum and its logarithm,
    then half a step each of |x - max| <= |lp| + ln z and of |lp|."""
    base = np.random.default_rng(vocab).standard_normal(vocab) * 2
    rows = [base + off for off in (0.0, 1e3, -1e3, 1e4, -1e4, 1e6, -1e6, 3e7)]
    rows += [np.full(vocab, LOW), np.full(vocab, 1e30), np.where(np.arange(vocab) % 3 == 0, -np.inf, base - 2e5)]
    x = torch.from_numpy(np.stack(rows)).float().to(DT[dt]).to(DEV)  # (the type's nearest: the lowest of bf16 too)
    x = torch.nan_to_num(x, neginf=-np.inf).repeat(repeat, 1) if dt == "f32" else x.repeat(repeat, 1)
    n = len(rows)
    tok = (np.arange(n * repeat) * 37 % vocab).astype(np.int32)
    lp, ent, top, tlp = md.md_token_logprobs(x, torch.from_numpy(tok).to(DEV), top_k=20)
    for r0 in {0, n * (repeat - 1)}:
        part = slice(r0, r0 + n)
        wlp, wtop, wtlp, lz = far_logprobs(host(x[part]), tok[part], 20)
        assert np.array_equal(top[part].cpu().numpy(), wtop)
        for got, want, size in ((host(lp[part]), wlp, lz), (host(tlp[part]), wtlp, lz[:, None])):
            assert np.array_equal(np.isneginf(got), np.isneginf(want))
            ok = np.isfinite(want)
            lim = plain.logprob_bound(np.where(ok, want, 0), size, 4)
            err = np.abs(np.where(ok, got - np.where(ok, want, 0), 0))
            assert (err <= lim).all(), [(r, float(err[r].max())) for r in range(n) if (err[r] > lim[r]).any()]
