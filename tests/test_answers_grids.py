"""Without a GPU: accumulated weights of sizes whose launch would pass the grid's 32 bits are refused."""
import ctypes
import os
import subprocess

from test_abi import lib  # noqa: F401  (the built library)
from test_answers_abi import UNS, mass
from test_sanitizers import ROOT


def test_padded_launch_of_a_step_is_refused(lib):  # noqa: F811
    """9 sequences of 2^20 heads are 9437184 workgroups, which whole rounds of the XCDs make 2^24."""
    heads = 1 << 20
    for B in (9, 15):
        a = mass(num_seqs=B, q_len=1, num_q_heads=heads, num_kv_heads=heads, max_kv_len=128, slot_stride=128,
                 q=1 << 56, k=2 << 56, lse=3 << 56, mass=4 << 56, slot_pos=5 << 56, kv_lens=6 << 56, pos0=6 << 56,
                 kv_stride_tok=heads * 64, kv_stride_blk=128 * heads * 64)
        assert lib.md_kv_mass(ctypes.byref(a), None) == UNS
        assert lib.md_kv_mass_workspace_bytes(ctypes.byref(a)) == 0


def test_grids_of_every_size_taken(tmp_path):
    exe = tmp_path / "driver"
    csrc = os.path.join(ROOT, "paper_2408_11049_amd", "csrc")
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "include"), "-I", csrc,
                    *[os.path.join(csrc, f) for f in ("plan.cpp", "plan_ops.cpp", "plan_answers.cpp")],
                    os.path.join(ROOT, "tests", "sanitize", "plan_grids_driver.cpp"), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "grids driver: ok" in r.stdout, r.stdout + r.stderr
