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


class OnGpu(torch.Tensor):
    """A host tensor that says it is on device 0, for host arithmetic on its sizes."""

    def get_device(self):
        return 0


def on_gpu(t):
    return t.as_subclass(OnGpu)


def test_sizes_past_32_bits_do_not_wrap(lib):  # noqa: F811
    """A bound, window or sink count past 32 bits is refused, not taken modulo 2^32."""
    cache = md.Kv4Cache(*map(on_gpu, md.kv4_empty(1, 16384, 1, 64, device="cpu")))
    q, lens = on_gpu(torch.zeros((1, 1, 4, 64))), on_gpu(torch.zeros(1, dtype=torch.int32))

    def need(**kw):
        return md.md_kv4_workspace_bytes(q, cache, lens, **kw)
    draft = dict(mode=md.MD_MODE_DRAFT)
    assert need() == need(max_kv_len=16384) > 0
    assert need(window=9000, **draft) > 0 == need(window=40, **draft)
    for wrap in (2 ** 32, -2 ** 32, 2 ** 40):
        for kw in (dict(max_kv_len=16384 + wrap), dict(max_kv_len=40 + wrap),
                   dict(window=9000 + wrap, **draft), dict(window=9000, n_sink=4 + wrap, **draft)):
            with pytest.raises(ValueError, match="32 bits"):
                need(**kw)
    for n_sink, window in ((4, 2 ** 32 + 40), (2 ** 32, 40)):
        with pytest.raises(ValueError, match="32 bits"):
            md.md_kv4_draft_attn(q, cache, lens, n_sink, window)


def test_caches_past_32_bits(lib):  # noqa: F811
    """Positions are 32-bit: a longer contiguous cache serves those it has, and a table of as
    many columns is refused."""
    far = 2 ** 32 + 96
    cache = [on_gpu(torch.zeros((1, 1, 1, w), dtype=torch.uint8).expand(1, far, 1, w))
             for w in (32, 32, 2, 2)]
    assert md.make_kv4_cache(cache).capacity == 2 ** 31 - 1
    pages = [on_gpu(torch.zeros((1, 16, 1, w), dtype=torch.uint8)) for w in (32, 32, 2, 2)]
    assert md.make_kv4_cache(pages, page_table=on_gpu(torch.zeros((1, 3), dtype=torch.int32))
                             ).max_pages_per_seq == 3

    class Wide(OnGpu):
        shape = property(lambda t: torch.Size((1, far)))
    with pytest.raises(ValueError, match="32 bits"):
        md.make_kv4_cache(pages, page_table=torch.zeros((1, 3), dtype=torch.int32).as_subclass(Wide))
