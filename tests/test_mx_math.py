"""How attention to a cache in 4 bits cuts heads into fragments, and to which XCD their workgroups go: compiled for the host alone, or in plain terms."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest

from paper_2507_08143_amd import build

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def M(tmp_path_factory):
    lib = str(tmp_path_factory.mktemp("mx_math") / "mx_math.so")
    subprocess.run([build.HIPCC, "-x", "hip", "--offload-host-only", "-std=c++17", "-O1", "-shared", "-fPIC",
                    "-I", build.INCLUDE, "-I", build.CSRC, os.path.join(HERE, "mx_math.cpp"), "-o", lib], check=True)
    return C.CDLL(lib)


@pytest.mark.parametrize("units", [32, 80, 256, 304])
@pytest.mark.parametrize("rows", [1, 16, 20, 40, 64])
def test_every_fragment_has_a_workgroup(M, units, rows):
    rng = np.random.default_rng(rows * 1000 + units)
    for heads in (1, 2, 3, 7, 8, 31, 96, 97, 128, 255, 256, 257, 384, 500, 512):
        for promised in (9, 16, 33, 141, 1000):
            launched = M.fragments_launched(heads, promised, rows, units)
            for steps in (np.full(heads, promised), rng.integers(max(1, promised - promised // 12), promised + 1, heads),
                          rng.integers(1, promised + 1, heads), np.full(heads, 7 * promised), np.ones(heads)):
                steps = np.ascontiguousarray(steps, dtype=np.int32)
                made = M.fragments_made(steps.ctypes.data_as(C.POINTER(C.c_int)), heads, promised, rows, units)
                assert heads <= made <= launched, (heads, promised, steps)


def test_the_parts_of_a_second_head_are_a_turn_of_its_own():
    """Part k of an odd head of P parts, behind one of Q: (k + Q % 8) % P where Q % 8 < P, else k.  Every part once, and at the XCD of the same part of the
    head before but for the Q % 8 that come round."""
    for P in range(1, 70):
        for Q in range(1, 70):
            turn = Q & 7
            parts = []
            for k in range(P):
                at = k + (turn if turn < P else 0)
                at -= P if at >= P else 0
                parts.append(at)
            assert sorted(parts) == list(range(P))
            if turn < P:
                apart = sum((Q + k) % 8 != p % 8 for k, p in enumerate(parts))
                assert apart <= turn


def test_pairs_of_heads_among_sixteen():
    for part in range(9):
        for heads in (1, 8, 15, 16, 17, 32, 100, 513):
            got = [(i & ~15) | (((i + (i >> 4) + part) & 7) << 1) | (i >> 3 & 1) if (i | 15) < heads else i for i in range(heads)]
            assert sorted(got) == list(range(heads))
            at = {h: i % 8 for i, h in enumerate(got)}
            assert all(at[h] == at[h + 1] for h in range(0, heads // 16 * 16, 2))
