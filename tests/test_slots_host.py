"""Bounds of the partials that attention launches leave in their workspaces (csrc/pq_plan.hpp), on the CPU: above what any launch plans, and growing
with the batch and the lengths."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    out = tmp_path_factory.mktemp("slotshost") / "libslots_host.so"
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-Wno-unknown-pragmas", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2502_00527_amd", "csrc"),
                    "-I", os.path.join(ROOT, "include"), os.path.join(ROOT, "tests", "host", "slots_host.cpp"), "-o", str(out)], check=True)
    return ctypes.CDLL(str(out))


@pytest.mark.parametrize("heads", [1, 2, 3, 7, 8, 32, 100, 300])
@pytest.mark.parametrize("group", [1, 4, 16])
@pytest.mark.parametrize("angles", [0, 1])
def test_partials_are_within_their_bounds(lib, heads, group, angles):
    rng = np.random.default_rng(heads)
    seqs = np.unique(np.concatenate([np.arange(1, 140), rng.integers(1, 3000, 40)])).astype(np.int32)
    pages = np.concatenate([np.arange(1, 300), rng.integers(1, 10000, 100)])
    lens = np.unique(np.concatenate([pages * 128, pages * 128 - 127, [2 ** 21, 2 ** 27]])).astype(np.int32)
    assert lib.slots_host(heads, group, angles, ctypes.c_void_p(seqs.ctypes.data), len(seqs), ctypes.c_void_p(lens.ctypes.data), len(lens)) == 0
