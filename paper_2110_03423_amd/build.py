"""Builds librsvd_gfx950.so from the HIP sources in csrc/ (hipcc, gfx950 only).

    python -m paper_2110_03423_amd.build

The library is placed next to this file so it travels with the source tree.
"""
import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "librsvd_gfx950.so")
OBJ_DIR = os.path.join(HERE, "_build")

SOURCES = ["sketch.hip", "gemm_f32.hip", "gemm_split_n.hip", "gemm_split_t.hip", "gemm_f64.hip", "gemm_f32acc64.hip", "chol.hip",
           "jacobi.hip", "apply.hip", "gram.hip", "rsvd_api.hip",
           "layer8_rows.hip", "layer8_gemm.hip", "layer8_grad.hip", "layer8_few.hip", "layer8_lowrank.hip", "layer8_api.hip",
           "dense.hip", "dense_nt_bf16.hip", "dense_nt_f16.hip", "dense_nt_f16_linear.hip", "dense_nt_f8.hip", "dense_nt_f8_exact.hip", "dense_kn_bf16.hip",
           "dense_kn_f16.hip", "gated.hip", "f8.hip", "orthogonal.hip", "dense_api.hip"]

# Packed fp32 instructions are switched off for device code on purpose.
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Wall", "-Wno-unused-function",
         "-Wno-pass-failed",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]


# Per-file additions.  chol.hip: its matrix-core accumulators are read by ordinary vector
# instructions after every update, so they must live in ordinary vector registers (the
# default puts them in the accumulation registers and copies them back and forth).
EXTRA_FLAGS = {"chol.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"]}


def _hipcc():
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", "hipcc"):
        if cand and (os.path.isabs(cand) and os.path.exists(cand) or not os.path.isabs(cand)):
            return cand
    raise RuntimeError("hipcc not found")


def _compile(src):
    obj = os.path.join(OBJ_DIR, os.path.splitext(src)[0] + ".o")
    cmd = [_hipcc()] + FLAGS + EXTRA_FLAGS.get(src, []) + ["-c", os.path.join(CSRC, src), "-o", obj]
    res = subprocess.run(cmd, capture_output=True, text=True)
    err = "\n".join(l for l in res.stderr.splitlines() if "packed-fp32-ops" not in l)
    if res.returncode != 0:
        raise RuntimeError(f"hipcc failed on {src}:\n{err}")
    return obj, err


def build_library(verbose=False, jobs=None):
    os.makedirs(OBJ_DIR, exist_ok=True)
    jobs = jobs or min(len(SOURCES), os.cpu_count() or 4)
    with ThreadPoolExecutor(max_workers=jobs) as ex:
        results = list(ex.map(_compile, SOURCES))
    if verbose:
        for _, err in results:
            if err.strip():
                print(err, file=sys.stderr)
    cmd = [_hipcc(), "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB] + [o for o, _ in results]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("link failed:\n" + res.stderr)
    return LIB


if __name__ == "__main__":
    print(build_library(verbose=True))
