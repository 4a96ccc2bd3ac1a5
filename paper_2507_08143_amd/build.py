"""Builds libcompactor.so (HIP, gfx950 only) in-tree next to this file.

    python -m paper_2507_08143_amd.build

hipcc cross-compiles without a GPU.  Objects go to _build/ at the repository
root (ignored by git); the shared library is written beside the Python binding
so that it travels with the source tree.
"""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD = os.path.join(ROOT, "_build")
LIB = os.path.join(HERE, "libcompactor.so")
SOURCES = ["api.hip", "gram.hip", "solve.hip", "score.hip", "select.hip", "gather.hip", "attention.hip",
           "cache.hip", "cache_attention.hip", "fp4.hip", "fp4_attention.hip", "rotate.hip", "pages.hip"]

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = [
    "-O3", "-std=c++17", "--offload-arch=gfx950", "-fPIC", "-fvisibility=hidden",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wno-unused-command-line-argument",
    "-I", INCLUDE, "-I", CSRC,
    '-DCOMPACTOR_API=__attribute__((visibility("default")))',
]


def _run(cmd):
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    out = "\n".join(l for l in r.stdout.splitlines()
                    if "packed-fp32-ops" not in l and "is not a recognized feature" not in l)
    if r.returncode != 0:
        raise RuntimeError("command failed: %s\n%s" % (" ".join(cmd), out))
    return out


def build(verbose: bool = False, jobs: int = 6, extra_flags=(), lib: str = LIB,
          build_dir: str = BUILD) -> str:
    """Compile every source and link `lib`.  extra_flags and a different
    output path serve experiments; the defaults give the product library."""
    os.makedirs(build_dir, exist_ok=True)
    objs = [os.path.join(build_dir, s.replace(".hip", ".o")) for s in SOURCES]

    def compile_one(pair):
        src, obj = pair
        return _run([HIPCC, *FLAGS, *extra_flags, "-c", os.path.join(CSRC, src), "-o", obj])

    with ThreadPoolExecutor(max_workers=jobs) as ex:
        outs = list(ex.map(compile_one, zip(SOURCES, objs)))
    out = _run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", *objs, "-o", lib])
    if verbose:
        print("\n".join(o for o in outs + [out] if o.strip()))
        print("built", lib)
    return lib


if __name__ == "__main__":
    build(verbose=True)
    sys.exit(0)
