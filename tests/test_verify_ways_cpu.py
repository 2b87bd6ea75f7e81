"""The rules for the verification of drafts (csrc/verify_plan.h), for the sizes of the GPU tests: a
rule that moves them off the kernels that they are for fails here."""
import os
import subprocess

import pytest

from tests import test_gpu_verify as V
from tests import test_gpu_verify_long as G

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ways(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("ways") / "verify_ways")
    subprocess.check_call(["g++", "-std=c++17", "-O2", "-Wall", "-I",
                           os.path.join(ROOT, "paper_2607_11985_amd", "csrc"),
                           os.path.join(ROOT, "tests", "verify_ways.cpp"), "-o", exe])

    def ask(sizes):
        """(how, short, parts, units, pieces, packs) of each (element, n, k, cols, draft)."""
        text = "".join(" ".join(str(int(v)) for v in s) + "\n" for s in sizes)
        out = subprocess.run([exe], input=text, text=True, capture_output=True,
                             check=True).stdout
        assert "wrong" not in out
        return [(w[0], *map(int, w[1:])) for w in map(str.split, out.splitlines())]
    return ask


@pytest.mark.parametrize("element", [2, 4])
@pytest.mark.parametrize("draft", [True, False])
def test_long_sizes_are_what_they_are_for(ways, element, draft):
    """Every size of test_gpu_verify_long.py, with the draft's scores and without."""
    for (n, k, cols), how in G.LONG.items():
        (got, *_), = ways([(element, n, k, cols, draft)])
        assert got == how[not draft], (n, k, cols)
    (_, is_short, *_), = ways([(2, *G.SHORT, draft)])
    assert is_short  # rows of fewer than 8 elements
    for how in ("read", "passed"):  # rows in one part and in several
        parts = [w[2] for w in ways([(2, *s, draft) for s in G.LONG]) if w[0] == how]
        assert 1 in parts and max(parts) > 1
    for size in G.GRAPHS:
        (got, *_), = ways([(element, *size, draft)])
        assert got == G.GRAPHS[size]


def test_sizes_of_the_gpu_tests_reach_every_kernel(ways):
    """All of test_gpu_verify.py's: both forms of long rows and of short ones, several parts, units and
    packs of a lane."""
    for element in (2, 4):
        found = ways([(element, *s, draft) for s in V.SIZES for draft in (True, False)])
        assert {"small", "read", "passed"} == {f[0] for f in found}
        assert {("small", 0), ("small", 1), ("passed", 0)} <= {f[:2] for f in found}
        assert any(f[0] == "read" and f[2] > 1 for f in found)
        assert any(f[0] == "read" and f[5] > 1 for f in found)
        assert any(f[0] == "passed" and f[5] > 1 for f in found)
    # the masked drafts there are read whole; those passed over are test_gpu_verify_long.py's
    assert {f[0] for f in ways([(4, *s, True) for s in [(4, 3, 70000), (64, 4, 33000)]])} == {"read"}


def test_short_rows_of_many_drafts_are_passed_over(ways):
    """total_kernel and draw_kernel take rows shorter than 16 bytes in that form alone."""
    for element in (2, 4):
        for cols in range(1, 16 // element):
            for draft in (False, True):
                found = ways([(element, n, k, cols, draft) for n in (1, 300, 10 ** 6)
                              for k in (*range(20, 70), 5000, 40000)])
                assert {f[0] for f in found} == {"small", "passed"}


def test_the_largest_sizes_have_a_plan(ways):
    """Up to 2^40 scores: within 64 parts and 4096 units, whatever their proportions."""
    for element in (2, 4):
        for draft in (False, True):
            ways([(element, 1, 0, 1 << 40, draft), (element, 1 << 40, 0, 1, draft),
                  (element, 1 << 20, 0, 1 << 20, draft), (element, 3, 1 << 30, 100, draft),
                  (element, 1 << 24, 100, 300, draft), (element, 7, 3, (1 << 32) + 5, draft)])
