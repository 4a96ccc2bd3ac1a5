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
            launched = [M.fragments_launched(heads, promised, rows, units, apart) for apart in (0, 1)]
            for steps in (np.full(heads, promised), rng.integers(max(1, promised - promised // 12), promised + 1, heads),
                          rng.integers(1, promised + 1, heads), np.full(heads, 7 * promised), np.ones(heads)):
                steps = np.ascontiguousarray(steps, dtype=np.int32)
                for apart in (0, 1):
                    made = M.fragments_made(steps.ctypes.data_as(C.POINTER(C.c_int)), heads, promised, rows, units, apart)
                    assert heads <= made <= launched[apart], (heads, promised, apart, steps)


def test_fragments_of_a_head(M):
    """The quotient by way of fp32, up to the most steps that a table has."""
    rng = np.random.default_rng(1)
    most = 2 ** 23
    for per in [1, 2, 3, 5, 7, 9, 31, 32, 33, 63, 64, 65, 127, 1000, 4097, 2 ** 20 + 1] + [int(x) for x in rng.integers(1, 10000, 50)]:
        for steps in [1, 2, per - 1, per, per + 1, most, most - 1] + [int(x) for x in rng.integers(1, most, 200)] + [per * int(k) + d for k in
                                                                                                                 rng.integers(1, max(2, most // per - 1), 40) for d in (-1, 0, 1)]:
            if 1 <= steps <= most:
                assert M.fragments_of(steps, per) == -(-steps // per), (steps, per)


def test_the_parts_of_two_heads_go_to_one_xcd():
    """Workgroup i takes part e(i) of the heads' parts, those of two neighbours in turn: every part of every head once, and the same parts of both at one XCD
    wherever the pairs before have an even number of parts."""
    rng = np.random.default_rng(0)
    for heads in (1, 2, 5, 8, 31, 64):
        for same in (True, False):
            for room in (0, 3, 40):
                parts = np.repeat(rng.integers(1, 12, (heads + 1) // 2), 2)[:heads] if same else rng.integers(1, 12, heads)
                total, first = int(parts.sum()), np.concatenate(([0], np.cumsum(parts)))
                grid = total + room
                seen, at = {}, {}
                for i in range(grid):
                    f = (i & ~15) | (i & 7) << 1 | (i >> 3 & 1) if (i | 15) < grid else i
                    assert 0 <= f < grid and f not in seen
                    seen[f] = None
                    if f >= total:
                        continue
                    h = int(np.searchsorted(first, f, side="right")) - 1
                    two = h & ~1
                    p0, p1 = int(parts[two]), int(parts[two + 1]) if two + 1 < heads else 0
                    q, both = f - int(first[two]), 2 * min(p0, p1)
                    head = two | (q & 1 if q < both else 1 if p1 > p0 else 0)
                    k = q >> 1 if q < both else q - both // 2
                    assert k < parts[head] and (head, k) not in at
                    at[head, k] = i % 8 if (i | 15) < grid else None
                assert len(at) == total
                if same:
                    for h in range(0, heads - 1, 2):
                        for k in range(int(parts[h])):
                            assert at[h, k] == at[h + 1, k]


def test_pairs_of_heads_among_sixteen():
    for part in range(9):
        for heads in (1, 8, 15, 16, 17, 32, 100, 513):
            got = [(i & ~15) | (((i + (i >> 4) + part) & 7) << 1) | (i >> 3 & 1) if (i | 15) < heads else i for i in range(heads)]
            assert sorted(got) == list(range(heads))
            at = {h: i % 8 for i, h in enumerate(got)}
            assert all(at[h] == at[h + 1] for h in range(0, heads // 16 * 16, 2))
