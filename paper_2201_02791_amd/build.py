"""Compile the HIP sources into ``libkge_mi355.so`` (gfx950 only), in-tree.

``python -m paper_2201_02791_amd.build`` builds; ``build(force=True)`` recompiles everything.
hipcc cross-compiles without a GPU, so this also runs on a CPU-only host.
"""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
OBJ = os.path.join(CSRC, "_build")
LIB = os.path.join(PKG, "libkge_mi355.so")
SOURCES = ["partition.hip", "gemm.hip", "gemm_bf16.hip", "rel_rows_bf16.hip", "rel_outer_bf16.hip", "gather.hip", "row_products.hip", "sampler_score.hip", "cgraph.hip", "optimizer.hip", "dropout.hip", "dense.hip", "dense_few.hip", "dense_rows_forward.hip", "dense_rows_input.hip", "norm.hip", "adamw.hip", "eval.hip", "api.hip"]
FLAGS = ["-O3", "-std=c++17", "-fPIC", "--offload-arch=gfx950", "-munsafe-fp-atomics",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-I" + os.path.join(ROOT, "include"), "-I" + CSRC, "-Wall", "-Wno-unused-function"]


def _stale(target, deps):
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = True) -> str:
    os.makedirs(OBJ, exist_ok=True)
    headers = [os.path.join(CSRC, "common.h"), os.path.join(CSRC, "sort_scan.h"), os.path.join(CSRC, "split_bf16.h"), os.path.join(CSRC, "split_f16.h"), os.path.join(CSRC, "dense.h"), os.path.join(CSRC, "dense_rows.h"), os.path.join(ROOT, "include", "kge_mi355.h"),
               os.path.join(ROOT, "include", "kge_mi355_testing.h")]

    def compile_one(src):
        s = os.path.join(CSRC, src)
        o = os.path.join(OBJ, src.replace(".hip", ".o"))
        if force or _stale(o, [s] + headers):
            cmd = ["hipcc"] + FLAGS + ["-c", s, "-o", o]
            if verbose:
                print("[build]", " ".join(cmd), flush=True)
            r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
            out = "\n".join(l for l in r.stdout.splitlines()
                            if "packed-fp32-ops" not in l and "is not a recognized feature" not in l)
            if r.returncode != 0:
                raise RuntimeError("hipcc failed for %s:\n%s" % (src, r.stdout))
            if verbose and out.strip():
                print(out, flush=True)
        return o

    with ThreadPoolExecutor(max_workers=min(5, os.cpu_count() or 1)) as ex:
        objs = list(ex.map(compile_one, SOURCES))
    if force or _stale(LIB, objs):
        cmd = ["hipcc", "-shared", "-fPIC", "--offload-arch=gfx950", "-o", LIB] + objs
        if verbose:
            print("[build]", " ".join(cmd), flush=True)
        subprocess.check_call(cmd)
    return LIB


if __name__ == "__main__":
    build(force="--force" in sys.argv)
    print(LIB)
