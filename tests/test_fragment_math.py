"""How long the fragments are that attention to a cache in 4 bits cuts heads into: none is left so long that the call waits for it.  Compiled for the host alone."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest

from paper_2507_08143_amd import build

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def M(tmp_path_factory):
    lib = str(tmp_path_factory.mktemp("fragment_math") / "fragment_math.so")
    subprocess.run([build.HIPCC, "-x", "hip", "--offload-host-only", "-std=c++17", "-O1", "-shared", "-fPIC",
                    "-I", build.INCLUDE, "-I", build.CSRC, os.path.join(HERE, "fragment_math.cpp"), "-o", lib], check=True)
    return C.CDLL(lib)


def _longest(M, steps, rows, apart):
    """Steps of the longest fragment on a device of 256 units."""
    steps = np.ascontiguousarray(steps, dtype=np.int32)
    return min(int(steps.max()), M.fragment_steps(steps.ctypes.data_as(C.POINTER(C.c_int)), len(steps), rows, 256, apart))


def _bound(steps):
    """What the rule wants: 32 steps a fragment (64 of heads of one length); or J fragments, a multiple of 256 above total / (0.375 sqrt(longest) + 1), of which the last ones
    of 512 heads take 320 at most and 96 at least are left: 0.375 J or more, so (0.375 sqrt(longest) + 1) / 0.375 steps and 1 for rounding; or, where those are
    more fragments than there are workgroups, 1536 at least, an equal share for each: a head of one length is cut into whole parts, and the last ones take theirs, so half
    of that and more, 512."""
    total, longest = int(steps.sum()), int(steps.max())
    return max(64, longest ** 0.5 + 4, total / 512 + 1)


@pytest.mark.parametrize("rows", [1, 4, 16, 20, 40, 64])
@pytest.mark.parametrize("apart", [0, 1])
@pytest.mark.parametrize("heads,long,steps,rest", [(512, 1, 1024, 1), (512, 1, 1024, 4), (512, 1, 400, 1), (448, 4, 256, 1), (416, 1, 1024, 1), (410, 2, 8192, 1),
                                                   (384, 1, 1024, 1), (256, 1, 1024, 1), (500, 1, 100, 1), (512, 9, 2000, 2), (300, 3, 700, 3), (64, 1, 400, 2)])
def test_a_long_head_among_short_ones(M, rows, apart, heads, long, steps, rest):
    s = np.full(heads, rest)
    s[heads // 2:heads // 2 + long] = steps
    assert _longest(M, s, rows, apart) <= _bound(s)


@pytest.mark.parametrize("rows", [1, 4, 16, 20, 40, 64])
@pytest.mark.parametrize("apart", [0, 1])
def test_any_lengths(M, rows, apart):
    rng = np.random.default_rng(rows)
    for heads in (1, 2, 7, 8, 31, 96, 128, 255, 256, 300, 384, 410, 448, 512):
        for most in (9, 30, 141, 1000, 8000):
            for s in (np.full(heads, most), rng.integers(1, most + 1, heads), np.exp(rng.uniform(0, np.log(most), heads)).astype(int) + 1,
                      np.where(rng.random(heads) < 3 / heads, most, 1)):
                assert _longest(M, s, rows, apart) <= _bound(s), (heads, most)
