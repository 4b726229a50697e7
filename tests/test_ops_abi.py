"""C ABI checks, without a GPU, of the 4-bit KV cache, sampled acceptance and the query/key
norm with rotation: struct layouts, refusals before any launch, workspace sizes, and the
host code under the sanitizers."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

import paper_2408_11049_amd as md
import plain_ops as plain
from test_abi import FAKE, lib  # noqa: F401  (the built library)
from test_sanitizers import ROOT, SAN, _runtime

INV, UNS, WS, OK = md.MD_ERR_INVALID_ARG, md.MD_ERR_UNSUPPORTED, md.MD_ERR_WORKSPACE, md.MD_OK
MAX = 2 ** 31 - 1


def cache(**over):
    c = md.MdKv4Cache()
    c.num_seqs, c.num_kv_heads, c.head_dim = 4, 2, 128
    c.k = c.v = c.k_scale = c.v_scale = FAKE
    c.stride_blk, c.stride_head, c.stride_tok = 2 * 96 * 64, 96 * 64, 64
    c.capacity = 96
    for k, v in over.items():
        setattr(c, k, v)
    return c


PAGED = dict(capacity=0, page_size=16, max_pages_per_seq=6, num_pages=30, page_table=FAKE)


def attn(**over):
    a = md.MdKv4AttnArgs()
    a.q_len, a.num_q_heads, a.dtype = 3, 8, md.MD_BF16
    a.q = a.o = a.kv_lens = FAKE
    a.max_kv_len = 96
    for k, v in over.items():
        setattr(a, k, v)
    return a


BAD_CACHE = [
    ("batch below 0", dict(num_seqs=-1), INV), ("no heads", dict(num_kv_heads=0), INV),
    ("head_dim 0", dict(head_dim=0), INV), ("head_dim 96", dict(head_dim=96), UNS),
    ("head_dim 256", dict(head_dim=256), UNS), ("no codes", dict(k=None), INV),
    ("no V scales", dict(v_scale=None), INV), ("codes misaligned", dict(v=FAKE + 8), INV),
    ("scales misaligned", dict(k_scale=FAKE + 2), INV),
    ("half rows apart", dict(stride_tok=32), INV), ("stride below 0", dict(stride_blk=-64), INV),
    ("tokens share rows", dict(stride_tok=0), INV), ("heads share rows", dict(stride_head=0), INV),
    ("token stride past 2^25", dict(stride_tok=(1 << 25) + 64), UNS),
    ("no capacity", dict(capacity=0), INV), ("table of a contiguous cache", dict(page_table=FAKE), INV),
    ("page size 12", dict(PAGED, page_size=12), INV), ("no table", dict(PAGED, page_table=None), INV),
    ("table misaligned", dict(PAGED, page_table=FAKE + 2), INV), ("no pages", dict(PAGED, num_pages=0), INV),
    ("page ids past int32", dict(PAGED, num_pages=1 << 31), INV),
    ("no table columns", dict(PAGED, max_pages_per_seq=0), INV),
    ("units past 2^31 - 1", dict(num_seqs=1 << 30), UNS),
]


@pytest.mark.parametrize("name,over,want", BAD_CACHE, ids=[b[0] for b in BAD_CACHE])
def test_bad_caches(lib, name, over, want):  # noqa: F811
    c = ctypes.byref(cache(**over))
    assert lib.md_kv4_append(c, 2, md.MD_BF16, FAKE, FAKE, FAKE, None, None) == want
    assert lib.md_kv4_read(c, 2, md.MD_F32, FAKE, FAKE, FAKE, None) == want
    if name != "no capacity":
        assert lib.md_kv4_verify_attn(c, ctypes.byref(attn()), None) == want
        assert lib.md_kv4_draft_attn(c, ctypes.byref(attn()), 4, 16, None) == want


def test_bad_rows(lib):  # noqa: F811
    c = ctypes.byref(cache())
    f, r = lib.md_kv4_append, lib.md_kv4_read
    assert f(None, 2, 1, FAKE, FAKE, FAKE, None, None) == INV
    assert f(c, -1, 1, FAKE, FAKE, FAKE, None, None) == INV
    assert f(c, 2, 2, FAKE, FAKE, FAKE, None, None) == INV
    assert f(c, 2, 1, None, FAKE, FAKE, None, None) == INV
    assert f(c, 2, 1, FAKE, FAKE + 8, FAKE, None, None) == INV
    assert f(c, 2, 1, FAKE, FAKE, None, None, None) == INV
    assert f(c, 2, 1, FAKE, FAKE, FAKE + 2, None, None) == INV
    assert f(c, 2, 1, FAKE, FAKE, FAKE, FAKE + 12, None) == INV      # lens_out over pos0
    assert f(c, 2, 1, FAKE, FAKE, FAKE, FAKE + 18, None) == INV
    assert f(c, MAX, 1, FAKE, FAKE, FAKE, None, None) == UNS         # rows past 2^31 - 1
    assert r(c, MAX, 1, FAKE, FAKE, FAKE, None) == UNS
    assert r(c, 2, 1, FAKE, FAKE, FAKE + 4, None) == INV
    assert r(c, 2, 1, None, FAKE, FAKE, None) == INV
    assert f(c, 0, 1, None, None, None, None, None) == OK            # nothing to do
    assert f(c, 0, 1, None, None, None, FAKE, None) == INV           # lengths alone, of what?
    assert f(c, 0, 1, None, None, FAKE, FAKE + 4, None) == INV
    assert f(ctypes.byref(cache(num_seqs=0)), 2, 1, None, None, None, FAKE, None) == OK
    assert r(ctypes.byref(cache(num_seqs=0, k=None)), 5, 1, None, None, None, None) == OK


BAD_ATTN = [
    ("q_len 0", dict(q_len=0), INV), ("q_len 17", dict(q_len=17), INV),
    ("heads no multiple", dict(num_q_heads=7), INV), ("no heads", dict(num_q_heads=0), INV),
    ("rows past 64", dict(num_q_heads=44), UNS), ("dtype", dict(dtype=3), INV),
    ("no q", dict(q=None), INV), ("no o", dict(o=None), INV), ("no lens", dict(kv_lens=None), INV),
    ("q misaligned", dict(q=FAKE + 8), INV), ("o misaligned", dict(o=FAKE + 8), INV),
    ("lse misaligned", dict(lse=FAKE + 2), INV), ("lens misaligned", dict(kv_lens=FAKE + 1), INV),
    ("bound below q_len", dict(max_kv_len=2), INV), ("bound past the cache", dict(max_kv_len=97), INV),
]


@pytest.mark.parametrize("name,over,want", BAD_ATTN, ids=[b[0] for b in BAD_ATTN])
@pytest.mark.parametrize("paged", [False, True])
def test_bad_attention(lib, name, over, want, paged):  # noqa: F811
    c, a = ctypes.byref(cache(**(PAGED if paged else {}))), ctypes.byref(attn(**over))
    assert lib.md_kv4_verify_attn(c, a, None) == want
    assert lib.md_kv4_draft_attn(c, a, 4, 16, None) == want
    if want == UNS:
        assert lib.md_kv4_workspace_bytes(c, a, md.MD_MODE_VERIFY, 0, 1) == 0


def test_attention_windows_and_workspaces(lib):  # noqa: F811
    c, a = ctypes.byref(cache()), ctypes.byref(attn())
    f = lib.md_kv4_draft_attn
    assert lib.md_kv4_verify_attn(c, None, None) == INV and lib.md_kv4_verify_attn(None, a, None) == INV
    assert f(c, a, -1, 4, None) == INV and f(c, a, 0, 0, None) == INV
    assert f(c, a, 0, 2 ** 31 - 60, None) == UNS and f(c, a, 2 ** 31 - 60, 1, None) == UNS
    assert lib.md_kv4_workspace_bytes(c, a, md.MD_MODE_DRAFT, 0, 0) == 0
    assert lib.md_kv4_workspace_bytes(c, a, 7, 0, 1) == 0
    long = dict(capacity=1 << 20, stride_head=64 << 20, stride_blk=128 << 20)
    far = dict(capacity=2 ** 31 - 20)
    assert lib.md_kv4_verify_attn(ctypes.byref(cache(**far)), ctypes.byref(attn(max_kv_len=2 ** 31 - 60)),
                                  None) == UNS
    need = [lib.md_kv4_workspace_bytes(ctypes.byref(cache(**long)), ctypes.byref(attn(max_kv_len=n)),
                                       md.MD_MODE_VERIFY, 0, 1) for n in (96, 1024, 8192, 1 << 20)]
    assert need[:2] == [0, 0] and 0 < need[2] <= need[3]  # a buffer for the longest serves all
    for ws, size in ((None, need[3]), (FAKE, need[3] - 1), (FAKE + 16, need[3])):
        big = attn(max_kv_len=1 << 20, workspace=ws, workspace_bytes=size)
        assert lib.md_kv4_verify_attn(ctypes.byref(cache(**long)), ctypes.byref(big), None) == WS
    assert lib.md_kv4_verify_attn(ctypes.byref(cache(num_seqs=1 << 22)), a, None) == UNS
    assert lib.md_kv4_verify_attn(ctypes.byref(cache(num_seqs=0, k=None)), ctypes.byref(attn(q=None)),
                                  None) == OK


def test_a_workspace_serves_every_smaller_context(lib):  # noqa: F811
    """Also where the longer call needs none itself (a workgroup per unit) and a shorter one is
    cut into ranges."""
    def need(B, n):
        c = cache(num_seqs=B, num_kv_heads=8, capacity=1 << 20, stride_head=64 << 20,
                  stride_blk=512 << 20)
        return lib.md_kv4_workspace_bytes(ctypes.byref(c), ctypes.byref(attn(num_q_heads=32, max_kv_len=n)),
                                          md.MD_MODE_VERIFY, 0, 1)
    for B in (1, 24, 32, 40, 48, 64, 96, 128, 1024, 1025):
        sizes = [need(B, n) for n in range(1000, 5000, 96)]
        assert sizes == sorted(sizes), B
    assert need(1024, 1 << 20) > 0 and need(1025, 1 << 20) == 0


def test_bad_sampled_acceptance(lib):  # noqa: F811
    def f(B=2, g=3, V=100, dt=0, p=FAKE, q=FAKE, d=FAKE, u=FAKE, a=FAKE, t=FAKE, ws=None, n=0):
        return lib.md_spec_accept(B, g, V, dt, p, q, d, u, a, t, ws, n, None)
    for bad in (dict(B=-1), dict(g=-1), dict(g=1024), dict(V=0), dict(V=(1 << 30) + 1), dict(dt=2),
                dict(p=None), dict(d=None), dict(u=None), dict(a=None), dict(t=None), dict(p=FAKE + 2),
                dict(q=FAKE + 1, dt=1), dict(d=FAKE + 2), dict(u=FAKE + 2), dict(a=FAKE + 1),
                dict(t=FAKE + 3)):
        assert f(**bad) == INV, bad
    assert f(B=1 << 22) == UNS
    assert f(B=0, p=None) == OK
    need = lib.md_spec_accept_workspace_bytes(2, 3, 128256)
    assert need > 0 and lib.md_spec_accept_workspace_bytes(2, 3, 1000) == 0
    assert lib.md_spec_accept_workspace_bytes(-1, 3, 128256) == 0
    for ws, n in ((None, need), (FAKE, need - 1), (FAKE + 8, need)):
        assert f(V=128256, ws=ws, n=n) == WS


def norm(**over):
    a = md.MdQkNormRopeArgs()
    a.num_seqs, a.n_new, a.num_q_heads, a.num_kv_heads, a.head_dim, a.dtype = 2, 3, 4, 2, 64, md.MD_BF16
    a.norm, a.eps, a.rot_dim, a.inv_freq, a.pos0 = 1, 1e-6, 64, FAKE, FAKE
    a.q, a.k_new, a.q_out, a.k_out = FAKE, FAKE + 0x10000, FAKE + 0x20000, FAKE + 0x30000
    a.q_stride_tok, a.q_stride_seq, a.k_stride_tok, a.k_stride_seq = 256, 768, 128, 384
    for k, v in over.items():
        setattr(a, k, v)
    return a


def kv(**over):
    c = md.MdKvCache()
    c.num_seqs, c.num_kv_heads, c.head_dim, c.dtype, c.capacity = 2, 2, 64, md.MD_BF16, 8
    c.k = c.v = FAKE + 0x90000
    c.kv_stride_tok, c.kv_stride_head, c.kv_stride_blk = 128, 64, 1024
    for k, v in over.items():
        setattr(c, k, v)
    return c


BAD_NORM = [
    dict(num_seqs=-1), dict(n_new=-1), dict(num_q_heads=0), dict(num_kv_heads=0), dict(dtype=5),
    dict(eps=-1.0), dict(eps=float("nan")), dict(norm=0, q_weight=FAKE), dict(rot_dim=8),
    dict(rot_dim=80), dict(rot_dim=-16), dict(q_stride_tok=-8), dict(k_stride_tok=4), dict(q=None),
    dict(k_new=None), dict(pos0=None), dict(q_out=None), dict(k_out=None), dict(v_new=FAKE + 0x40000),
    dict(inv_freq=None), dict(inv_freq=FAKE + 2), dict(q=FAKE + 8), dict(k_weight=FAKE + 8),
    dict(pos0=FAKE + 2), dict(lens_out=FAKE + 4), dict(lens_out=FAKE + 0x50002),
    dict(q_out=FAKE + 16), dict(q_out=FAKE + 0x10010), dict(k_out=FAKE + 0x10010),
    dict(k_out=FAKE + 0x20010), dict(q_out=FAKE, q_stride_tok=264, q_stride_seq=792),
]


@pytest.mark.parametrize("over", BAD_NORM, ids=[str(i) for i in range(len(BAD_NORM))])
def test_bad_norm(lib, over):  # noqa: F811
    assert lib.md_qk_norm_rope(ctypes.byref(norm(**over)), None, None) == INV


def test_bad_norm_caches_and_sizes(lib):  # noqa: F811
    f = lib.md_qk_norm_rope
    assert f(None, None, None) == INV
    assert f(ctypes.byref(norm(head_dim=96, rot_dim=0)), None, None) == UNS
    assert f(ctypes.byref(norm(num_seqs=1 << 20, n_new=1 << 12)), None, None) == UNS
    assert f(ctypes.byref(norm(num_q_heads=65537)), None, None) == UNS
    assert f(ctypes.byref(norm(n_new=0, q=None)), None, None) == OK
    assert f(ctypes.byref(norm(n_new=0, lens_out=FAKE + 4)), None, None) == INV
    assert f(ctypes.byref(norm(n_new=0, lens_out=FAKE, pos0=None)), None, None) == INV
    assert f(ctypes.byref(norm(num_seqs=0, lens_out=FAKE, pos0=None)), None, None) == OK
    with_v = norm(v_new=FAKE + 0x40000, v_stride_tok=128, v_stride_seq=384)
    for over in (dict(num_seqs=3), dict(num_kv_heads=1), dict(head_dim=128), dict(dtype=0), dict(k=None),
                 dict(v=FAKE + 8), dict(capacity=0), dict(kv_stride_tok=4)):
        assert f(ctypes.byref(with_v), ctypes.byref(kv(**over)), None) == INV, over
    assert f(ctypes.byref(norm()), ctypes.byref(kv()), None) == INV  # a cache, no V rows
    big = norm(q_stride_seq=2 ** 62 + 8, q_stride_tok=2 ** 62 + 8, q_out=FAKE + 0x10000)
    assert f(ctypes.byref(big), None, None) == INV                   # overlaps; no overflow


def test_struct_layouts(tmp_path):
    """The binding's structs against the header's, by a C compiler."""
    structs = {"md_kv4_cache": md.MdKv4Cache, "md_kv4_attn_args": md.MdKv4AttnArgs,
               "md_qk_norm_rope_args": md.MdQkNormRopeArgs}
    lines = []
    for name, s in structs.items():
        lines.append(f'printf("%zu\\n", sizeof({name}));')
        lines += [f'printf("%zu\\n", offsetof({name}, {f}));' for f, _ in s._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "magicdec.h"\nint main(void) {\n'
                   + "\n".join(lines) + "\nreturn 0; }\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src),
                    "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    want = []
    for s in structs.values():
        want.append(ctypes.sizeof(s))
        want += [getattr(s, f).offset for f, _ in s._fields_]
    assert got == want


@pytest.mark.skipif(_runtime("libasan.so") is None, reason="gcc's AddressSanitizer runtime is not installed")
def test_plans_under_sanitizers(tmp_path):
    exe = tmp_path / "driver"
    csrc = os.path.join(ROOT, "paper_2408_11049_amd", "csrc")
    subprocess.run(["g++", "-std=c++17", "-O1", *SAN, "-I", os.path.join(ROOT, "include"), "-I", csrc,
                    os.path.join(csrc, "plan.cpp"), os.path.join(csrc, "plan_ops.cpp"),
                    os.path.join(ROOT, "tests", "sanitize", "plan_ops_driver.cpp"), "-o", str(exe)],
                   check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300,
                       env={**os.environ, "ASAN_OPTIONS": "detect_leaks=1:abort_on_error=0"})
    assert r.returncode == 0 and "plan ops driver: ok" in r.stdout, r.stdout + r.stderr


# ---- the references themselves ----

def test_reference_rounding_is_nearest():
    """No level is nearer than the one chosen, and ties go to the even code; scales follow
    a / 2^e < 7."""
    rng = np.random.default_rng(1)
    x = np.concatenate([rng.standard_normal((64, 64)) * np.exp2(rng.integers(-20, 20, (64, 1))),
                        np.full((1, 64), 7.0), np.full((1, 64), 6.999), np.full((1, 64), 3.5)])
    codes, scales = plain.kv4_round(x)
    v = plain.kv4_values(codes, scales)
    step = np.repeat(np.exp2(scales - 127.0), 32, -1)
    every = np.concatenate([plain.LEVELS, -plain.LEVELS])
    best = np.abs(x[..., None] - every * step[..., None]).min(-1)
    assert np.array_equal(np.abs(x - v), best)
    top = np.abs(x).reshape(len(x), 2, 32).max(-1) / np.exp2(scales - 127.0)
    assert (top < 7).all() and (top >= 3.5).all()
    assert v[-3, 0] == 8.0 and v[-2, 0] == 6.0 and v[-1, 0] == 3.0 or v[-1, 0] == 4.0


def test_reference_accept_is_speculative_sampling():
    """Over all outcomes of a small case the first token's probability is the target's."""
    p, q = np.array([0.5, 0.125, 0.25, 0.125]), np.array([0.125, 0.5, 0.25, 0.125])
    n = 64
    prob = np.zeros(4)
    for d in range(4):
        grid = (np.arange(n) + 0.5) / n
        u = np.stack(np.meshgrid(grid, grid, indexing="ij"), -1).reshape(-1, 2)
        B = len(u)
        _, tok = plain.spec_accept(np.tile(p, (B, 2, 1)), np.tile(q, (B, 1, 1)),
                                   np.full((B, 1), d), u)
        prob += q[d] * np.bincount(tok[:, 0], minlength=4) / B
    assert np.allclose(prob, p, atol=1e-12)
