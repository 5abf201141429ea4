"""In which form a pass of attention counts its units of work: the host's rule, compiled by itself."""
import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    d = tmp_path_factory.mktemp("units")
    src, lib = d / "units.cpp", d / "units.so"
    src.write_text('#include "%s"\nextern "C" int by_warps(long long e, long long h, long long t, int s) { return asx::runs_by_warps(e, h, t, s); }\n'
                   'extern "C" int fit(long long e, long long h, long long t, int s) { return asx::units_fit(e, h, t, s); }\n'
                   % os.path.join(ROOT, "paper_2210_15458_b200", "csrc", "as_units.h"))
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-o", str(lib), str(src)])
    L = ctypes.CDLL(str(lib))
    for f in (L.by_warps, L.fit):
        f.argtypes = [ctypes.c_longlong] * 3 + [ctypes.c_int]
    return L


@pytest.mark.parametrize("entries,heads,tokens", [
    (30000, 8, 1 << 20), (1, 512, 1 << 30), (3750 * 8, 8, 1 << 20), (1 << 20, 64, 1 << 12), (512, 1, 1 << 28), (513, 1, (1 << 27) + 1), (64, 8, 1 << 27),
    (64, 8, (1 << 27) - 32), (128, 8, 8192), (1, 1, 1), (100000, 8, 8192), (511, 1, 64)])
@pytest.mark.parametrize("behind_shared", [0, 1])
def test_units_of_the_form_that_is_taken_fit_31_bits(rule, entries, heads, tokens, behind_shared):
    """Whatever the entry point accepts (units of 128 tokens fit), the units of the form that is taken fit too."""
    accepted = entries * heads * -(-tokens // 128) < 1 << 31
    assert bool(rule.fit(entries, heads, tokens, 7)) == accepted
    warps = bool(rule.by_warps(entries, heads, tokens, behind_shared))
    small = entries * heads * -(-tokens // 32) < 1 << 31
    assert warps == (small and (bool(behind_shared) or entries * heads >= 512))
    if accepted:
        assert entries * heads * -(-tokens // (32 if warps else 128)) < 1 << 31
