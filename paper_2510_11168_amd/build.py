"""Builds libelmo_head.so (HIP, gfx950 only) in-tree with hipcc."""
from __future__ import annotations

import os
import subprocess
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libelmo_head.so")
SOURCES = [os.path.join(HERE, "csrc", s) for s in ("elmo_head.hip", "elmo_lm.hip")]
HEADERS = [os.path.join(HERE, "csrc", h) for h in ("errors.h", "numerics.h", "tiles.h", "kernels.h", "topk_levels.h", "plan.h", "topk.h",
                                                   "rows.h", "norm.h", "int8.h", "sample.h", "distill.h")] + [
    os.path.join(os.path.dirname(HERE), "include", "elmo_head.h")]

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
    # packed FP32 instructions are kept out of the generated code on purpose
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # the update arithmetic rounds after every FP32 operation: no contraction into fused multiply-adds
    "-ffp-contract=off",
    "-Wno-unused-result",
]


def _hipcc(args: list[str], verbose: bool) -> None:
    cmd = [os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), *args]
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + res.stdout + res.stderr)


def build(verbose: bool = False) -> str:
    """Compile unconditionally, the sources side by side; returns the path of the shared library."""
    flags = [f for f in HIPCC_FLAGS if f != "-shared"]
    with tempfile.TemporaryDirectory() as tmp:
        objects = [os.path.join(tmp, os.path.basename(s) + ".o") for s in SOURCES]
        with ThreadPoolExecutor(len(SOURCES)) as pool:
            list(pool.map(lambda so: _hipcc([*flags, "-c", so[0], "-o", so[1]], verbose), zip(SOURCES, objects)))
        _hipcc(["--offload-arch=gfx950", "-fPIC", "-shared", *objects, "-o", LIB_PATH], verbose)
    return LIB_PATH


def is_built() -> bool:
    return os.path.exists(LIB_PATH)


if __name__ == "__main__":
    print(build(verbose=True))
