"""The Python functions of the 4-bit KV cache, sampled acceptance and the query/key norm
with rotation, without a GPU: what they make of their arguments before the library is called."""
import pytest
import torch

import paper_2408_11049_amd as md
from test_abi import lib  # noqa: F401  (the built library)


def host_call(name):
    """A call's arguments, by the documented names and in their order, on the CPU."""
    cache = md.kv4_empty(1, 8, 1, 64, device="cpu")
    rows = torch.zeros((1, 2, 1, 64))
    lens = torch.zeros(1, dtype=torch.int32)
    return {
        "md_kv4_append": dict(cache=cache, k_new=rows, v_new=rows, pos0=lens),
        "md_kv4_read": dict(cache=cache, pos0=lens, n=2),
        "md_kv4_verify_attn": dict(q=rows, cache=cache, kv_lens=lens),
        "md_kv4_draft_attn": dict(q=rows, cache=cache, kv_lens=lens, n_sink=1, window=4),
        "md_spec_accept": dict(target_probs=torch.ones((1, 2, 8)), draft_probs=None,
                               draft=lens[None], u=torch.zeros((1, 2))),
        "md_qk_norm_rope": dict(q=rows, k_new=rows, pos0=lens, inv_freq=torch.ones(32)),
    }[name]


CALLS = ["md_kv4_append", "md_kv4_read", "md_kv4_verify_attn", "md_kv4_draft_attn",
         "md_spec_accept", "md_qk_norm_rope"]


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


@pytest.mark.parametrize("name", [c for c in CALLS if "kv4" in c])
def test_a_cache_of_four_tensors(lib, name):  # noqa: F811
    """A cache may be any sequence of the four tensors."""
    kw = host_call(name)
    for kind in (tuple, list):
        with pytest.raises(ValueError, match="on a GPU"):
            getattr(md, name)(**{**kw, "cache": kind(kw["cache"])})
