"""Sampled acceptance, without a GPU: buffers that share memory.  The kernels write tokens and
accepted while other workgroups still read the drafts, so a call whose outputs or workspace
overlap an input or each other is refused; one where they only touch is not."""
import pytest

import paper_2408_11049_amd as md
from test_abi import lib  # noqa: F401  (the built library)

BASE, GAP = 1 << 40, 1 << 32  # addresses, never dereferenced: without a GPU no launch succeeds
B, G, V = 3, 4, 128256


def sizes(dtype, sampled):
    es = 2 if dtype == md.MD_BF16 else 4
    return dict(p=B * (G + 1) * V * es, q=B * G * V * es if sampled else 0, draft=B * G * 4,
                u=B * (G + 1) * 4, accepted=B * 4, tokens=B * (G + 1) * 4)


def call(lib, dtype, at, sampled, need):  # noqa: F811
    return lib.md_spec_accept(B, G, V, dtype, at["p"], at["q"] if sampled else None, at["draft"],
                              at["u"], at["accepted"], at["tokens"], at["ws"], need, None)


@pytest.mark.parametrize("dtype", [md.MD_F32, md.MD_BF16])
@pytest.mark.parametrize("sampled", [True, False])
def test_buffers_that_share_memory(lib, dtype, sampled):  # noqa: F811
    need = lib.md_spec_accept_workspace_bytes(B, G, V)
    size = dict(sizes(dtype, sampled), ws=need)
    apart = {name: BASE + i * GAP for i, name in enumerate(size)}
    outs, ins = ("accepted", "tokens", "ws"), ("p", "q", "draft", "u")
    unit = 256  # every alignment at once
    for i, out in enumerate(outs):
        for other in ins + outs[i + 1:]:
            if not size[other]:
                continue
            # The same start, the output's last bytes over the first, its first over the last.
            for shift in {0, -((size[out] - 1) // unit * unit), (size[other] - 1) // unit * unit}:
                at = dict(apart)
                at[out] = at[other] + shift
                assert call(lib, dtype, at, sampled, need) == md.MD_ERR_INVALID_ARG, (out, other, shift)


@pytest.mark.parametrize("dtype", [md.MD_F32, md.MD_BF16])
def test_neighbours_and_shared_inputs(lib, dtype):  # noqa: F811
    """Buffers one behind the other, and inputs that are one buffer, are the caller's right; the
    launch then fails for want of a GPU only."""
    import torch
    if torch.cuda.is_available():
        pytest.skip("the addresses are made up")
    need = lib.md_spec_accept_workspace_bytes(B, G, V)
    size = dict(sizes(dtype, True), ws=need)
    at, end = {}, BASE
    for name in ("ws", "tokens", "accepted", "draft", "u", "p", "q"):
        at[name], end = end, end + size[name]
    assert call(lib, dtype, at, True, need) == md.MD_ERR_HIP
    at["q"] = at["p"]  # probabilities of draft and target in one tensor
    assert call(lib, dtype, at, True, need) == md.MD_ERR_HIP
    at["q"] = at["tokens"]  # not looked at where the drafts have no probabilities
    assert call(lib, dtype, at, False, need) == md.MD_ERR_HIP
