"""The Python functions of shared prefixes, accumulated weights, eviction and token log
probabilities, without a GPU: what they make of their arguments before the library is called."""
import numpy as np
import pytest
import torch

import paper_2408_11049_amd as md
import plain_answers as plain
from test_abi import lib  # noqa: F401  (the built library)


def host_call(name):
    """A call's arguments, by the documented names and in their order, on the CPU."""
    q = torch.zeros((2, 3, 4, 64))
    kv, pre = torch.zeros((2, 20, 2, 64)), torch.zeros((1, 30, 2, 64))
    lens, one = torch.zeros(2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    mass, pos = torch.zeros((2, 2, 20)), torch.zeros((2, 2, 20), dtype=torch.int32)
    return {
        "md_prefix_attn": dict(q=q, k=kv, v=kv, kv_lens=lens, prefix_k=pre, prefix_v=pre, prefix_lens=one),
        "md_prefix_workspace_bytes": dict(q=q, k=kv, v=kv, kv_lens=lens, prefix_k=pre, prefix_v=pre,
                                          prefix_lens=one),
        "md_kv_mass": dict(q=q, k=kv, kv_lens=lens, lse=torch.zeros((2, 3, 4)), mass=mass, slot_pos=pos, pos0=lens),
        "md_kv_evict": dict(k=kv, v=kv.clone(), mass=mass, slot_pos=pos, kv_lens=lens, seq_lens=lens, budget=10),
        "md_token_logprobs": dict(logits=torch.zeros((2, 50)), tokens=lens),
    }[name]


CALLS = ["md_prefix_attn", "md_prefix_workspace_bytes", "md_kv_mass", "md_kv_evict", "md_token_logprobs"]


@pytest.mark.parametrize("name", CALLS)
def test_arguments_by_name(lib, name):  # noqa: F811
    """Every argument can be given by its name, the first one too: each way the call gets as far
    as refusing host tensors."""
    f, kw = getattr(md, name), host_call(name)
    first = next(iter(kw))
    for args, named in ((tuple(kw.values()), {}), ((kw[first],), {k: kw[k] for k in kw if k != first}),
                        ((), kw)):
        with pytest.raises(ValueError, match="on a GPU"):
            f(*args, **named)
    with pytest.raises(TypeError, match=first):  # and a missing one is named
        f(**{k: kw[k] for k in kw if k != first})


def test_short_names():
    assert md.prefix_attn is md.md_prefix_attn and md.kv_mass is md.md_kv_mass
    assert md.kv_evict is md.md_kv_evict and md.token_logprobs is md.md_token_logprobs


class OnGpu(torch.Tensor):
    """A host tensor that says it is on device 0, for the checks of sizes and types."""

    def get_device(self):
        return 0


def on_gpu(kw, **over):
    kw = {**kw, **over}
    return {k: t.as_subclass(OnGpu) if isinstance(t, torch.Tensor) else t for k, t in kw.items()}


I32 = torch.int32
BAD = [
    ("md_prefix_workspace_bytes", dict(prefix_k=torch.zeros((1, 30, 2, 64), dtype=torch.bfloat16)), "dtype"),
    ("md_prefix_workspace_bytes", dict(prefix_v=torch.zeros((1, 31, 2, 64))), "equal shapes"),
    ("md_prefix_workspace_bytes", dict(prefix_v=torch.zeros((1, 30, 2, 64), dtype=torch.bfloat16)), "share a dtype"),
    ("md_prefix_workspace_bytes", dict(prefix_k=torch.zeros((1, 30, 1, 64))), "heads and head_dim"),
    ("md_prefix_workspace_bytes", dict(prefix_lens=torch.zeros(1, dtype=torch.int64)), "prefix_lens"),
    ("md_prefix_workspace_bytes", dict(prefix_lens=torch.zeros(2, dtype=I32)), "hold max_prefix_len"),
    ("md_prefix_workspace_bytes", dict(max_prefix_len=31), "hold max_prefix_len"),
    ("md_prefix_workspace_bytes", dict(max_kv_len=2 ** 32 + 10), "32 bits"),
    ("md_prefix_workspace_bytes", dict(prefix_page_table=torch.zeros((1, 4), dtype=torch.int64)), "prefix_page_table"),
    ("md_prefix_workspace_bytes", dict(prefix_page_table=torch.zeros((0, 4), dtype=I32)), "prefix_page_table"),
    ("md_prefix_workspace_bytes", dict(prefix_page_table=torch.zeros((1, 4), dtype=I32), max_prefix_len=2 ** 33),
     "32 bits"),
    ("md_kv_mass", dict(q=torch.zeros((2, 3, 4, 128))[..., ::2]), "contiguous"),
    ("md_kv_mass", dict(k=torch.zeros((2, 20, 2, 64), dtype=torch.bfloat16)), "dtype"),
    ("md_kv_mass", dict(lse=torch.zeros((2, 4, 3))), "lse"),
    ("md_kv_mass", dict(pos0=torch.zeros(2)), "pos0"),
    ("md_kv_mass", dict(mass=torch.zeros((2, 2, 21))), "slots"), ("md_kv_mass", dict(mass=torch.zeros((2, 1, 20))), "slots"),
    ("md_kv_mass", dict(slot_pos=torch.zeros((2, 2, 20))), "slots"), ("md_kv_mass", dict(max_kv_len=21), "hold max_kv_len"),
    ("md_kv_mass", dict(page_table=torch.zeros((2, 2))), "page_table"),
    ("md_kv_mass", dict(page_table=torch.zeros((2, 2), dtype=I32), max_kv_len=2 ** 32 + 5), "32 bits"),
    ("md_token_logprobs", dict(tokens=torch.zeros(2, dtype=torch.int64)), "tokens"),
    ("md_token_logprobs", dict(tokens=torch.zeros(3, dtype=I32)), "tokens"),
    ("md_token_logprobs", dict(logits=torch.zeros((2, 100))[:, ::2]), "unit-stride"),
    ("md_token_logprobs", dict(logits=torch.zeros((2, 3, 50))[:, :2], tokens=None), "one stride"),
    ("md_token_logprobs", dict(tokens=None, logprobs=torch.zeros(2)), "without tokens"),
    ("md_token_logprobs", dict(top_k=2 ** 32 + 1), "32 bits"),
]


# Refused as well, but where tensors are truly on a GPU.
BAD_ON_GPU = [
    ("md_kv_mass", dict(kv_lens=torch.zeros(1, dtype=I32)), "kv_lens"),
    ("md_kv_mass", dict(accepted=torch.zeros(2, dtype=torch.int64)), "accepted"),
    ("md_kv_evict", dict(kv_lens=torch.zeros(2, dtype=torch.int64)), "kv_lens"),
    ("md_kv_evict", dict(seq_lens=torch.zeros(1, dtype=I32)), "seq_lens"),
    ("md_kv_evict", dict(budget=2 ** 32 + 10), "32 bits"),
    ("md_kv_evict", dict(n_sink=2 ** 32), "32 bits"),
    ("md_kv_evict", dict(recent=-2 ** 32), "32 bits"),
    ("md_kv_evict", dict(lens_out=torch.zeros(2)), "lens_out"),
    ("md_kv_evict", dict(mass=torch.zeros((2, 2, 40))[:, :, ::2]), "slots"),
    ("md_token_logprobs", dict(logprobs=torch.zeros(3)), "logprobs"),
    ("md_token_logprobs", dict(top_k=2, top=torch.zeros((2, 2))), "top"),
]


@pytest.mark.parametrize("name,over,match", BAD, ids=[f"{b[0]}-{i}" for i, b in enumerate(BAD)])
def test_malformed_tensors(lib, name, over, match):  # noqa: F811
    with pytest.raises(ValueError, match=match):
        f = getattr(md, name)
        md._torch()
        getattr(f, "__wrapped__", f)(**on_gpu(host_call(name), **over))


def test_a_prefix_workspace_from_tensors(lib):  # noqa: F811
    kw = on_gpu(host_call("md_prefix_workspace_bytes"))
    assert md.md_prefix_workspace_bytes(**kw) > 0
    assert md.md_prefix_workspace_bytes(**kw, max_kv_len=20, max_prefix_len=30) == md.md_prefix_workspace_bytes(**kw)


# ---- the references themselves ----

def test_reference_of_a_prefix_is_attention_over_both():
    """The prefix and the own tokens as one cache, by another formula."""
    rng = np.random.default_rng(0)
    lens, plens, L, Hq, Hkv, d = [3, 9], [5], 3, 4, 2, 8
    q = rng.standard_normal((2, L, Hq, d))
    own = [[rng.standard_normal((n, Hkv, d)) for n in lens] for _ in "kv"]
    pre = [[rng.standard_normal((n, Hkv, d)) for n in plens] for _ in "kv"]
    o, lse = plain.prefix_attention(q, *own, lens, *pre, plens, 0.3)[:2]
    for b, n in enumerate(lens):
        for i in range(L):
            for h in range(Hq):
                k, v = (np.concatenate([pre[x][0][:, h // 2], own[x][b][: n - L + i + 1, h // 2]]) for x in (0, 1))
                w = np.exp(0.3 * k @ q[b, i, h])
                assert np.allclose(o[b, i, h], w @ v / w.sum()) and np.isclose(lse[b, i, h], np.log(w.sum()))


def test_reference_of_weights_sums_softmax_columns():
    rng = np.random.default_rng(1)
    n, L, d = 7, 2, 8
    q, k = rng.standard_normal((1, L, 2, d)), rng.standard_normal((n, 1, d))
    s = np.einsum("ihd,jd->ihj", q[0], k[:, 0]) / np.sqrt(d)
    s[0, :, n - 1] = -np.inf                              # the first row is one token behind
    lse = np.log(np.exp(s).sum(2))[None]
    want = np.exp(s - lse[0][..., None]).sum((0, 1))
    want[: n - L] += 0.5
    m, pos, err = plain.kv_mass(q, [k], [n], lse, np.full((1, 1, n + 1), 0.5), np.full((1, 1, n + 1), -3), [40])
    assert np.allclose(m[0, 0, :n], want) and m[0, 0, n] == 0.5 and (err >= 0).all()
    assert pos[0, 0].tolist() == [-3] * (n - L) + [40, 41, -3]


def test_reference_of_eviction_by_hand():
    mass = np.array([[[5.0, 1.0, 4.0, 0.5, 3.0, 2.0]]])
    pos = np.array([[[9, 0, 8, 7, 6, 10]]])
    rows = np.arange(6)[None, None].repeat(1, 0)
    # Budget 3, one sink (slot 1 at position 0), the newest of 11 (slot 5 at position 10): they stay with
    # the heaviest, slot 0; slots 1 and 0 are in place, slot 5 moves to 2.
    r, m, p, n = plain.evict(rows, mass, pos, [6], [11], 3, 1, 1)
    assert n.tolist() == [3] and r[0, 0, :3].tolist() == [0, 1, 5]
    assert m[0, 0, :3].tolist() == [5.0, 1.0, 2.0] and p[0, 0, :3].tolist() == [9, 0, 10]
    assert r[0, 0, 3:].tolist() == [3, 4, 5]              # what is behind the budget stays as it was


def test_reference_of_logprobs_by_hand():
    x = np.log(np.array([[0.5, 0.25, 0.25], [1.0, 1.0, 1.0]]))
    x[1] = [-np.inf, 3.0, -np.inf]
    lp, ent, top, tlp, _ = plain.token_logprobs(x, np.array([2, -1]), 2)
    assert np.allclose(lp, [np.log(0.25), 0.0]) and np.allclose(ent, [1.5 * np.log(2), 0.0])
    assert top.tolist() == [[0, 1], [1, 0]] and np.allclose(tlp[0], np.log([0.5, 0.25])) and tlp[1, 1] == -np.inf
