"""Builds ``libht.so`` (the C-ABI CUDA library) in-tree with nvcc for sm_100a.

Run as ``python -m paper_2404_12022_b200.build``; ``build()`` is also what
``__graft_entry__.build()`` calls.  nvcc cross-compiles, so no GPU is needed.
"""
from __future__ import annotations

import concurrent.futures
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libht.so")
SOURCES = ["ht_api.cu", "transfer.cu", "transfer_tc.cu", "attn_simt.cu", "verify.cu", "compact.cu", "draft.cu", "rope.cu", "norm_rope.cu", "attn_static.cu"]
# compiled once per shape of the attention scores (plain, capped, biased, both) or per type of the logits: (source, macro, its values)
SPLIT = [("sample.cu", "HT_SAMPLE_DTYPE", (2, 1, 0)), ("attn_tc_pair.cu", "HT_ATTN_SHAPE", (3, 2, 1, 0)), ("attn_tc.cu", "HT_ATTN_SHAPE", (3, 2, 1, 0))]
# (source, object, flags), what takes longest first
UNITS = ([(src, "%s_%d.o" % (src[:-3], i), ["-D%s=%d" % (macro, i)]) for src, macro, values in SPLIT for i in values]
         + [(src, src[:-3] + ".o", []) for src in SOURCES])
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC", "--expt-relaxed-constexpr", "--compress-mode=size"]


def _nvcc() -> str:
    cand = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "bin", "nvcc")
    return cand if os.path.exists(cand) else "nvcc"


def _newest_header() -> float:
    times = [os.path.getmtime(os.path.join(CSRC, f)) for f in os.listdir(CSRC) if f.endswith((".cuh", ".h"))]
    times.append(os.path.getmtime(os.path.join(HERE, "..", "include", "ht.h")))
    return max(times)


def _compile(unit, verbose: bool) -> str:
    src, name, flags = unit
    obj = os.path.join(OBJ, name)
    path = os.path.join(CSRC, src)
    if os.path.exists(obj) and os.path.getmtime(obj) > max(os.path.getmtime(path), _newest_header()):
        return obj
    cmd = [_nvcc(), *NVCC_FLAGS, *flags, "-c", path, "-o", obj]
    if verbose:
        cmd.insert(1, "-Xptxas=-v")
    res = subprocess.run(cmd, capture_output=True, text=True)
    if verbose or res.returncode:
        sys.stderr.write(res.stdout + res.stderr)
    if res.returncode:
        raise RuntimeError("nvcc failed on " + src)
    return obj


def build(force: bool = False, verbose: bool = False) -> str:
    os.makedirs(OBJ, exist_ok=True)
    if force:
        for f in os.listdir(OBJ):
            os.remove(os.path.join(OBJ, f))
    with concurrent.futures.ThreadPoolExecutor(max_workers=len(UNITS)) as pool:
        objs = list(pool.map(lambda u: _compile(u, verbose), UNITS))
    if (not os.path.exists(LIB)) or any(os.path.getmtime(o) > os.path.getmtime(LIB) for o in objs):
        tmp = LIB + ".tmp%d" % os.getpid()
        subprocess.run([_nvcc(), "-shared", "-o", tmp, *objs, "-gencode", "arch=compute_100a,code=sm_100a"],
                       check=True)
        os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
