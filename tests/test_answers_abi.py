"""C ABI checks, without a GPU, of attention over a shared prefix, accumulated weights, eviction
and token log probabilities: struct layouts, refusals before any launch, workspace sizes, and
the host code under the sanitizers."""
import ctypes
import os
import subprocess

import pytest

import paper_2408_11049_amd as md
from test_abi import FAKE, lib  # noqa: F401  (the built library)
from test_sanitizers import ROOT, SAN, _runtime

INV, UNS, WS, OK = md.MD_ERR_INVALID_ARG, md.MD_ERR_UNSUPPORTED, md.MD_ERR_WORKSPACE, md.MD_OK
MAX = 2 ** 31 - 1
STEP = 1 << 32                      # far from one another
A, B_, C, D, E, F = (FAKE + i * STEP for i in range(6))


def filled(struct, over):
    for k, v in over.items():
        setattr(struct, k, v)
    return struct


# ---- attention over a shared prefix ----

def attn(**over):
    a = md.MdAttnArgs()
    a.num_seqs, a.q_len, a.num_q_heads, a.num_kv_heads, a.head_dim, a.dtype = 4, 2, 8, 2, 128, md.MD_BF16
    a.q = a.k = a.v = a.o = a.kv_lens = FAKE
    a.kv_stride_blk, a.kv_stride_tok, a.kv_stride_head = 96 * 256, 256, 128
    a.max_kv_len = 96
    return filled(a, over)


def prefix(**over):
    p = md.MdPrefix()
    p.num_prefixes = 2
    p.k = p.v = p.lens = FAKE
    p.kv_stride_blk, p.kv_stride_tok, p.kv_stride_head = 500 * 256, 256, 128
    p.max_len = 500
    return filled(p, over)


OWN_PAGES = dict(page_size=16, max_pages_per_seq=6, num_pages=30, page_table=FAKE)
PRE_PAGES = dict(page_size=16, max_pages_per_prefix=32, num_pages=90, page_table=FAKE)

BAD_PREFIX = [
    # over the attention's arguments, over the prefix's, the status
    ("no q", dict(q=None), {}, INV), ("no o", dict(o=None), {}, INV), ("no k", dict(k=None), {}, INV),
    ("no v", dict(v=None), {}, INV), ("no lens", dict(kv_lens=None), {}, INV),
    ("no prefix k", {}, dict(k=None), INV), ("no prefix v", {}, dict(v=None), INV),
    ("no prefix lens", {}, dict(lens=None), INV), ("no prefixes", {}, dict(num_prefixes=0), INV),
    ("prefixes below 0", {}, dict(num_prefixes=-2), INV), ("no divisor", {}, dict(num_prefixes=3), INV),
    ("more prefixes than sequences", {}, dict(num_prefixes=8), INV), ("max_len below 0", {}, dict(max_len=-1), INV),
    ("dtype", dict(dtype=2), {}, INV), ("head_dim 96", dict(head_dim=96), {}, UNS),
    ("heads no multiple", dict(num_q_heads=7), {}, INV), ("q_len 0", dict(q_len=0), {}, INV),
    ("rows past 64", dict(q_len=17), {}, INV), ("rows past 64 by heads", dict(num_q_heads=66), {}, UNS),
    ("bound below q_len", dict(max_kv_len=1), {}, INV),
    ("q misaligned", dict(q=FAKE + 8), {}, INV), ("prefix k misaligned", {}, dict(k=FAKE + 8), INV),
    ("prefix lens misaligned", {}, dict(lens=FAKE + 2), INV), ("lse misaligned", dict(lse=FAKE + 2), {}, INV),
    ("error word misaligned", dict(err_word=FAKE + 2), {}, INV),
    ("stride below 0", {}, dict(kv_stride_blk=-256), INV), ("rows off 16 bytes", {}, dict(kv_stride_tok=260), INV),
    ("heads share rows", {}, dict(kv_stride_head=64), INV), ("own heads share rows", dict(kv_stride_head=64), {}, INV),
    ("token stride past 2^28", {}, dict(kv_stride_tok=(1 << 28) + 8), UNS),
    ("page size 12", {}, dict(PRE_PAGES, page_size=12), INV), ("no table", {}, dict(PRE_PAGES, page_table=None), INV),
    ("a table of contiguous rows", {}, dict(page_table=FAKE), INV),
    ("table misaligned", {}, dict(PRE_PAGES, page_table=FAKE + 2), INV), ("no pages", {}, dict(PRE_PAGES, num_pages=0), INV),
    ("too few columns", {}, dict(PRE_PAGES, max_pages_per_prefix=31), INV),
    ("page ids past int32", {}, dict(PRE_PAGES, num_pages=1 << 31), INV),
    ("own page size 12", dict(OWN_PAGES, page_size=12), {}, INV),
    ("own columns too few", dict(OWN_PAGES, max_pages_per_seq=5), {}, INV),
    ("bound past what can be addressed", {}, dict(max_len=MAX), UNS),
    ("rows past 2^31", dict(num_seqs=1 << 27), {}, UNS),
    ("no workspace", {}, {}, WS), ("short workspace", dict(workspace=FAKE, workspace_bytes=1024), {}, WS),
    ("workspace misaligned", dict(workspace=FAKE + 128, workspace_bytes=1 << 40), {}, WS),
]


@pytest.mark.parametrize("name,over,pover,want", BAD_PREFIX, ids=[b[0] for b in BAD_PREFIX])
def test_bad_prefix(lib, name, over, pover, want):  # noqa: F811
    a, p = ctypes.byref(attn(**over)), ctypes.byref(prefix(**pover))
    assert lib.md_prefix_attn(a, p, None) == want
    if want == UNS:
        assert lib.md_prefix_workspace_bytes(a, p) == 0


def test_prefix_of_nothing(lib):  # noqa: F811
    a, p = ctypes.byref(attn()), ctypes.byref(prefix())
    assert lib.md_prefix_attn(None, p, None) == INV and lib.md_prefix_attn(a, None, None) == INV
    assert lib.md_prefix_workspace_bytes(None, p) == 0 == lib.md_prefix_workspace_bytes(a, None)
    none = attn(num_seqs=0, q=None, o=None, k=None, v=None, kv_lens=None)
    assert lib.md_prefix_attn(ctypes.byref(none), p, None) == OK


@pytest.mark.parametrize("over", [dict(), dict(num_seqs=64, q_len=5, num_q_heads=32, num_kv_heads=8),
                                  dict(dtype=md.MD_F32, num_seqs=16, head_dim=64), dict(num_seqs=2, q_len=1)])
def test_prefix_workspace_serves_shorter_calls(lib, over):  # noqa: F811
    """A buffer for one pair of bounds serves every smaller pair."""
    lens = [0, 1, 127, 128, 129, 255, 256, 257, 1000, 5000, 8192, 33000, 70000]

    def need(own, pre):
        return lib.md_prefix_workspace_bytes(ctypes.byref(attn(**over, max_kv_len=own)),
                                             ctypes.byref(prefix(max_len=pre)))
    grid = [[need(max(own, 5), pre) for pre in lens] for own in lens]
    assert grid[0][0] > 0
    for i in range(len(lens)):
        for j in range(len(lens)):
            assert i == 0 or grid[i][j] >= grid[i - 1][j], (lens[i], lens[j])
            assert j == 0 or grid[i][j] >= grid[i][j - 1], (lens[i], lens[j])


# ---- accumulated weights ----

def mass(**over):
    a = md.MdKvMassArgs()
    a.num_seqs, a.q_len, a.num_q_heads, a.num_kv_heads, a.head_dim, a.dtype = 4, 3, 8, 2, 64, md.MD_BF16
    a.q, a.k, a.lse, a.mass, a.slot_pos = A, B_, C, D, E
    a.kv_lens = a.pos0 = F
    a.kv_stride_blk, a.kv_stride_tok, a.kv_stride_head = 200 * 128, 128, 64
    a.max_kv_len, a.slot_stride = 200, 210
    return filled(a, over)


MASS_PAGES = dict(page_size=32, max_pages_per_seq=7, num_pages=50, page_table=F + 4096)
BAD_MASS = [
    ("batch below 0", dict(num_seqs=-1), INV), ("q_len 0", dict(q_len=0), INV), ("no heads", dict(num_kv_heads=0), INV),
    ("heads no multiple", dict(num_q_heads=9), INV), ("dtype", dict(dtype=5), INV), ("head_dim 0", dict(head_dim=0), INV),
    ("head_dim 96", dict(head_dim=96), UNS), ("bound below q_len", dict(max_kv_len=2), INV),
    ("slots below the bound", dict(slot_stride=199), INV),
    *[(f"no {n}", {n: None}, INV) for n in ("q", "k", "kv_lens", "lse", "pos0", "mass", "slot_pos")],
    *[(f"{n} misaligned", {n: F + 0x1002}, INV) for n in ("kv_lens", "lse", "pos0", "mass", "slot_pos", "accepted")],
    ("q misaligned", dict(q=A + 8), INV), ("k misaligned", dict(k=B_ + 8), INV),
    ("rows off 16 bytes", dict(kv_stride_tok=132), INV), ("heads share rows", dict(kv_stride_head=32), INV),
    ("stride below 0", dict(kv_stride_tok=-128), INV), ("token stride past 2^28", dict(kv_stride_tok=(1 << 28) + 8), UNS),
    ("page size 12", dict(MASS_PAGES, page_size=12), INV), ("no table", dict(MASS_PAGES, page_table=None), INV),
    ("too few columns", dict(MASS_PAGES, max_pages_per_seq=6), INV), ("no pages", dict(MASS_PAGES, num_pages=0), INV),
    ("rows past 2^30", dict(q_len=1 << 29, max_kv_len=1 << 29, slot_stride=1 << 29), UNS),
    ("bound past what can be addressed", dict(max_kv_len=MAX, slot_stride=1 << 33), UNS),
    ("key blocks past 31 bits", dict(max_kv_len=2 ** 31 - 256, slot_stride=1 << 33), UNS),
    ("workgroups past 2^24", dict(num_seqs=1 << 23), UNS),
    ("mass is slot_pos", dict(slot_pos=D), INV), ("mass over the lse", dict(lse=D + 4), INV),
    ("mass among the keys", dict(mass=B_ + 1024), INV), ("slot_pos over pos0", dict(slot_pos=F), INV),
    ("mass over q", dict(mass=A + 64), INV),
    ("mass over the table", dict(MASS_PAGES, mass=F + 4096), INV),
    ("a prompt without its workspace", dict(q_len=200), WS),
    ("a short one", dict(q_len=200, workspace=FAKE + 9 * STEP, workspace_bytes=256), WS),
    ("misaligned", dict(q_len=200, workspace=FAKE + 9 * STEP + 64, workspace_bytes=1 << 40), WS),
    ("over mass", dict(q_len=200, workspace=D, workspace_bytes=1 << 20), INV),
]


@pytest.mark.parametrize("name,over,want", BAD_MASS, ids=[b[0] for b in BAD_MASS])
def test_bad_mass(lib, name, over, want):  # noqa: F811
    assert lib.md_kv_mass(ctypes.byref(mass(**over)), None) == want


def test_mass_of_nothing_and_workspaces(lib):  # noqa: F811
    def f(**over):
        return lib.md_kv_mass_workspace_bytes(ctypes.byref(mass(**over)))
    assert lib.md_kv_mass(None, None) == INV and lib.md_kv_mass_workspace_bytes(None) == 0
    assert lib.md_kv_mass(ctypes.byref(mass(num_seqs=0, q=None, mass=None)), None) == OK
    assert f() == 0 == f(q_len=64) and f(q_len=65) > 0        # parts of 256 rows of a KV head at least
    assert f(head_dim=96) == 0 == f(q_len=0)
    long = dict(num_seqs=1, q_len=4096, max_kv_len=4096, slot_stride=4096)
    assert f(**long) % (2 * 4096 * 4) == 0


# ---- eviction ----

def cache(**over):
    c = md.MdKvCache()
    c.num_seqs, c.num_kv_heads, c.head_dim, c.dtype = 4, 2, 64, md.MD_BF16
    c.k, c.v = A, B_
    c.kv_stride_blk, c.kv_stride_tok, c.kv_stride_head = 200 * 128, 128, 64
    c.capacity = 200
    return filled(c, over)


EVICT = dict(mass=C, slot_pos=D, slot_stride=200, lens=E, seq_lens=E + 4096, budget=100, n_sink=4, recent=50,
             lens_out=F, workspace=None, workspace_bytes=0)


def evict(lib, c=None, **over):  # noqa: F811
    kw = {**EVICT, **over}
    return lib.md_kv_evict(None if c is None else ctypes.byref(c), *kw.values(), None)


CACHE_PAGES = dict(capacity=0, page_size=16, max_pages_per_seq=13, num_pages=60, page_table=E + 8192)
BAD_EVICT = [
    ("no head_dim", dict(head_dim=0), {}, INV),
    ("head_dim 96", dict(head_dim=96, kv_stride_head=96, kv_stride_tok=192), {}, UNS),
    ("dtype", dict(dtype=4), {}, INV), ("no k", dict(k=None), {}, INV), ("v misaligned", dict(v=B_ + 8), {}, INV),
    ("no capacity", dict(capacity=0), {}, INV), ("heads share rows", dict(kv_stride_head=32), {}, INV),
    ("page size 12", dict(CACHE_PAGES, page_size=12), {}, INV), ("no table", dict(CACHE_PAGES, page_table=None), {}, INV),
    ("no pages", dict(CACHE_PAGES, num_pages=0), {}, INV), ("page ids past int32", dict(CACHE_PAGES, num_pages=1 << 31), {}, INV),
    ("units past 2^22", dict(num_seqs=1 << 22), {}, UNS),
    *[(f"no {n}", {}, {n: None}, INV) for n in ("mass", "slot_pos", "lens", "seq_lens")],
    *[(f"{n} misaligned", {}, {n: F + 0x1002}, INV) for n in ("mass", "slot_pos", "lens", "seq_lens", "lens_out")],
    ("budget 0", {}, dict(budget=0), INV), ("no slots", {}, dict(slot_stride=0), INV),
    ("slots past what can be addressed", {}, dict(slot_stride=MAX), UNS),
    ("slots whose successors are", {}, dict(slot_stride=2 ** 31 - 2048), UNS),
    ("sinks below 0", {}, dict(n_sink=-1), INV), ("recent below 0", {}, dict(recent=-1), INV),
    ("more held than kept", {}, dict(n_sink=60, recent=41), INV),
    ("held past 32 bits", {}, dict(n_sink=MAX, recent=MAX), INV),
    ("mass is slot_pos", {}, dict(slot_pos=C), INV), ("lens_out is lens", {}, dict(lens_out=E), INV),
    ("lens_out is seq_lens", {}, dict(lens_out=E + 4096), INV), ("lens_out over mass", {}, dict(lens_out=C + 8), INV),
    ("mass among the keys", {}, dict(mass=A + 256), INV), ("lens among the values", {}, dict(lens=B_ + 256), INV),
    ("mass over the table", CACHE_PAGES, dict(mass=E + 8192), INV),
    ("many moves, no workspace", dict(capacity=5000), dict(slot_stride=5000, budget=1000), WS),
    ("many moves, a short one", dict(capacity=5000), dict(slot_stride=5000, budget=1000, workspace=FAKE + 9 * STEP,
                                                          workspace_bytes=512), WS),
    ("a misaligned one", dict(capacity=5000), dict(slot_stride=5000, budget=1000, workspace=FAKE + 9 * STEP + 8,
                                                   workspace_bytes=1 << 40), WS),
    ("one over lens", dict(capacity=5000), dict(slot_stride=5000, budget=1000, workspace=E, workspace_bytes=1 << 20), INV),
]


@pytest.mark.parametrize("name,over,call,want", BAD_EVICT, ids=[b[0] for b in BAD_EVICT])
def test_bad_evict(lib, name, over, call, want):  # noqa: F811
    assert evict(lib, cache(**over), **call) == want


def test_evict_of_nothing_and_workspaces(lib):  # noqa: F811
    assert evict(lib) == INV
    assert evict(lib, cache(num_seqs=0, k=None), mass=None) == OK
    assert evict(lib, cache(num_seqs=0), budget=0) == INV
    f = lib.md_kv_evict_workspace_bytes

    def need(slots, budget, **over):
        return f(ctypes.byref(cache(capacity=8192, **over)), slots, budget)
    assert f(None, 100, 10) == 0 == need(0, 10) == need(100, 0) == need(8192, 512)
    assert need(8192, 513) == 256 + 33024 == need(1 << 20, 513)  # 8 * 513 pairs of 8 bytes; the cache holds 8192
    assert need(8192, 8000) == 0 == need(8192, 9000)                 # at most 192 moves, and none


# ---- log probabilities ----

LOGP = dict(rows=6, vocab=1000, row_stride=1000, dtype=md.MD_F32, logits=A, tokens=B_, top_k=5, logprobs=C,
            entropy=D, top=E, top_logprobs=F, workspace=None, workspace_bytes=0)


def logp(lib, **over):  # noqa: F811
    return lib.md_token_logprobs(*{**LOGP, **over}.values(), None)


BAD_LOGP = [
    ("rows below 0", dict(rows=-1), INV), ("vocab 0", dict(vocab=0), INV), ("vocab past 2^30", dict(vocab=(1 << 30) + 1), INV),
    ("rows overlap", dict(row_stride=999), INV), ("stride below 0", dict(rows=1, row_stride=-1), INV),
    ("dtype", dict(dtype=2), INV), ("top_k -1", dict(top_k=-1), INV), ("top_k 33", dict(top_k=33), INV),
    ("rows past 2^22", dict(rows=1 << 22), UNS), ("no logits", dict(logits=None), INV),
    ("logits misaligned", dict(logits=A + 2), INV), ("half logits misaligned", dict(logits=A + 1, dtype=md.MD_BF16), INV),
    ("tokens alone", dict(logprobs=None), INV), ("logprobs alone", dict(tokens=None), INV), ("no top", dict(top=None), INV),
    ("no top_logprobs", dict(top_logprobs=None), INV), ("a top of none", dict(top_k=0, top_logprobs=None), INV),
    *[(f"{n} misaligned", {n: B_ + 0x1002}, INV) for n in ("tokens", "logprobs", "entropy", "top", "top_logprobs")],
    ("logprobs is entropy", dict(entropy=C), INV), ("top over tokens", dict(top=B_ + 8), INV),
    ("entropy among the logits", dict(entropy=A + 12000), INV),
    ("segments without a workspace", dict(vocab=5000, row_stride=5000), WS),
    ("a short one", dict(vocab=5000, row_stride=5000, workspace=FAKE + 9 * STEP, workspace_bytes=16), WS),
    ("a misaligned one", dict(vocab=5000, row_stride=5000, workspace=FAKE + 9 * STEP + 4, workspace_bytes=1 << 40), WS),
    ("one over the logits", dict(vocab=5000, row_stride=5000, workspace=A + 256, workspace_bytes=1 << 20), INV),
]


@pytest.mark.parametrize("name,over,want", BAD_LOGP, ids=[b[0] for b in BAD_LOGP])
def test_bad_logprobs(lib, name, over, want):  # noqa: F811
    assert logp(lib, **over) == want


def test_logprobs_of_nothing_and_workspaces(lib):  # noqa: F811
    assert logp(lib, rows=0, logits=None) == OK and logp(lib, rows=0, vocab=0) == INV
    f = lib.md_token_logprobs_workspace_bytes
    assert f(6, 4096, 5) == 0 < f(6, 4097, 5) < f(6, 4097, 32)
    assert f(-1, 5000, 5) == 0 == f(6, 0, 5) == f(6, 5000, 33)
    assert f(1, 1 << 30, 32) < 256 * (32 * 8 + 12) + 1024           # at most 256 segments a row


# ---- the binding's structs and the host code ----

def test_struct_layouts(tmp_path):
    """The binding's structs against the header's, by a C compiler."""
    structs = {"md_prefix": md.MdPrefix, "md_kv_mass_args": md.MdKvMassArgs}
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
                    *[os.path.join(csrc, f) for f in ("plan.cpp", "plan_ops.cpp", "plan_answers.cpp")],
                    os.path.join(ROOT, "tests", "sanitize", "plan_answers_driver.cpp"), "-o", str(exe)],
                   check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300,
                       env={**os.environ, "ASAN_OPTIONS": "detect_leaks=1:abort_on_error=0"})
    assert r.returncode == 0 and "plan answers driver: ok" in r.stdout, r.stdout + r.stderr
