"""Attention over a shared prefix and token log probabilities on the GPU, where calls end: waves without work,
sizes of nothing, values far from zero."""
import numpy as np
import pytest
import torch

import paper_2408_11049_amd as md
from test_gpu_answers import DEV, check_logp, rand

pytestmark = pytest.mark.gpu


# ---- log probabilities ----

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
