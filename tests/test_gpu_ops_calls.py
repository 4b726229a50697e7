"""The step operators' functions by every way their arguments can be given: by place, by name,
a cache as a plain sequence, on a stream: the same results, bit for bit."""
import pytest
import torch

import paper_2408_11049_amd as md

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def made(seed=0):
    g = torch.Generator().manual_seed(seed)

    def rand(*shape, dtype=torch.bfloat16):
        return torch.randn(shape, generator=g).to(dtype).to(DEV)
    B, n, Hq, Hkv, d, V = 3, 2, 4, 2, 64, 70001
    cache = md.kv4_empty(B, 2000, Hkv, d, device=DEV)
    for t in cache:
        t.zero_()
    lens = torch.tensor([5, 700, 1998], dtype=torch.int32, device=DEV)
    q, k, v = rand(B, n, Hq, d), rand(B, n, Hkv, d), rand(B, n, Hkv, d)
    md.md_kv4_append(cache, rand(B, 1500, Hkv, d), rand(B, 1500, Hkv, d), torch.zeros_like(lens))
    probs = [rand(B, m, V, dtype=torch.float32).softmax(-1) for m in (n + 1, n)]
    return {
        "md_kv4_append": dict(cache=cache, k_new=k, v_new=v, pos0=lens),
        "md_kv4_read": dict(cache=cache, pos0=lens, n=3),
        "md_kv4_verify_attn": dict(q=q, cache=cache, kv_lens=lens),
        "md_kv4_draft_attn": dict(q=q, cache=cache, kv_lens=lens, n_sink=3, window=1500),
        "md_spec_accept": dict(target_probs=probs[0], draft_probs=probs[1],
                               draft=torch.randint(0, V, (B, n), generator=g).to(torch.int32).to(DEV),
                               u=torch.rand((B, n + 1), generator=g).to(DEV)),
        "md_qk_norm_rope": dict(q=q, k_new=k, pos0=lens, inv_freq=torch.rand(d // 2, generator=g).to(DEV)),
    }


@pytest.mark.parametrize("name", ["md_kv4_append", "md_kv4_read", "md_kv4_verify_attn",
                                  "md_kv4_draft_attn", "md_spec_accept", "md_qk_norm_rope"])
def test_ways_to_call(name):
    f, kw = getattr(md, name), made()[name]
    print(f"[calls] {name}", flush=True)

    def results(*args, **named):
        r = f(*args, **named)
        torch.cuda.synchronize()
        state = list(kw["cache"]) if "cache" in kw else []
        return [t.clone() for t in (list(r) if isinstance(r, tuple) else [r]) + state]
    want = results(*kw.values())
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    ways = [results(**kw), results(stream=side, **kw), results(*kw.values(), stream=side)]
    if "cache" in kw:
        for kind in (tuple, list):
            ways.append(results(**{**kw, "cache": kind(kw["cache"])}))
    with torch.cuda.stream(side):
        ways.append(results(**kw))
    for got in ways:
        assert len(got) == len(want) and all(torch.equal(a, b) for a, b in zip(got, want))
