"""Without a GPU: the cases of tests/prefix_wide_cases.py reach the tiles that waves share, in as many parts as they say, and their
inputs tell a key too few, too many or counted twice from a rounding."""
import os
import subprocess

import numpy as np
import pytest
import torch

from prefix_wide_cases import CASES, Inputs, edges
from test_sanitizers import ROOT


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    exe = tmp_path_factory.mktemp("plan") / "driver"
    csrc = os.path.join(ROOT, "paper_2408_11049_amd", "csrc")
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "include"), "-I", csrc,
                    *[os.path.join(csrc, f) for f in ("plan.cpp", "plan_ops.cpp", "plan_answers.cpp")],
                    os.path.join(ROOT, "tests", "sanitize", "plan_prefix_driver.cpp"), "-o", str(exe)], check=True)
    return str(exe)


@pytest.mark.parametrize("name", CASES)
def test_plan_of_the_case(driver, name):
    (Hq, Hkv, d, L, n, page, ppage, bound, plens), parts = CASES[name]
    out = subprocess.run([driver, *map(str, (n * len(plens), len(plens), L, Hq, Hkv, d, page, ppage, bound))],
                         capture_output=True, text=True, check=True).stdout
    assert out.split() == ["1", str(parts)]
    assert max(plens) <= bound


@pytest.mark.parametrize("name,prefixes", [("one part, 240 rows, 64 channels, pages of 8", (2, 16, 29)),
                                           ("sixteen parts, 288 rows", (0,)), ("eight parts, 200 rows", (1,))])
def test_wrong_keys_are_told_from_roundings(name, prefixes):
    """The oracle with one key left out, one counted twice, or a key of zeros behind the last: at every edge some row
    is out of its bounds on o, and some on lse."""
    case = Inputs(name)
    for p in prefixes:
        k, v, T = case.pk[p], case.pv[p], case.plens[p]
        o, lse, ob, lb = case.oracle(p)

        def beyond(k, v):
            o2, l2 = case.oracle(p, k, v)[:2]
            return bool((np.abs(o2 - o) > ob).any() and (np.abs(l2 - lse) > lb).any())
        for j in edges(T, case.parts):
            keep = torch.arange(T) != j
            assert beyond(k[keep], v[keep]), ("left out", T, j)
            assert beyond(torch.cat([k, k[j:j + 1]]), torch.cat([v, v[j:j + 1]])), ("twice", T, j)
        assert beyond(torch.cat([k, 0 * k[:1]]), torch.cat([v, 0 * v[:1]])), ("zeros", T)
