"""Builds the HIP library in-tree: paper_2107_06876_amd/liblcn_hip.so (gfx950)."""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "liblcn_hip.so")

# translation unit -> extra flags
SOURCES = {
    "kernels_structure.hip": ["-ffp-contract=off"],   # bucket rule: separate multiply and add
    "kernels_factors.hip": [],
    "kernels_mfma.hip": [],
    "kernels_sweep_mid.hip": [],
    "kernels_sweep_short.hip": [],
    "kernels_sweep_long.hip": [],
    "kernels_iter.hip": [],
    "kernels_nystrom.hip": [],
    "kernels_dense.hip": [],
    "kernels_buckets.hip": [],
    "kernels_batched.hip": ["-ffp-contract=off"],  # bucket rule again
    "kernels_planes.hip": [],
    "kernels_linear.hip": [],
    "kernels_gated.hip": [],
    "kernels_gated_narrow.hip": [],
    "kernels_norm.hip": [],
    "kernels_orthogonal.hip": [],
    "kernels_pair.hip": [],
    "kernels_entropy.hip": [],
    "kernels_attention_f32.hip": [],
    "kernels_attention_bf16.hip": [],
    "kernels_attention_grad_f32.hip": [],
    "kernels_attention_grad_bf16.hip": [],
    "attention_api.hip": [],
    "lcn_api.hip": [],
    "calibrate.hip": [],
}

COMMON = ["--offload-arch=gfx950", "-O3", "-fPIC", "-std=c++17", "-I" + os.path.join(ROOT, "include"), "-I" + CSRC,
          "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-Wno-unused-command-line-argument"]


def _hipcc():
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", "hipcc"):
        if cand and (os.path.sep not in cand or os.path.exists(cand)):
            return cand
    raise RuntimeError("hipcc not found")


def build_library(force: bool = True, verbose: bool = False) -> str:
    hipcc = _hipcc()
    objdir = os.path.join(HERE, "_build")
    os.makedirs(objdir, exist_ok=True)
    headers = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".h")]
    headers.append(os.path.join(ROOT, "include", "lcn.h"))
    newest_header = max(os.path.getmtime(h) for h in headers)
    jobs = []
    objs = []
    for src, extra in SOURCES.items():
        path = os.path.join(CSRC, src)
        if not os.path.exists(path):
            continue
        obj = os.path.join(objdir, src + ".o")
        objs.append(obj)
        stale = force or not os.path.exists(obj) or os.path.getmtime(obj) < max(os.path.getmtime(path), newest_header)
        if stale:
            jobs.append([hipcc, "-c", path, "-o", obj] + COMMON + extra)

    def run(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        res = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
        if res.returncode != 0:
            raise RuntimeError("hipcc failed:\n" + " ".join(cmd) + "\n" + res.stdout)
        return res.stdout

    with ThreadPoolExecutor(max_workers=8) as ex:
        for out in ex.map(run, jobs):
            if verbose and out.strip():
                print(out)
    if jobs or not os.path.exists(LIB):
        tmp = LIB + ".tmp%d" % os.getpid()
        run([hipcc, "-shared", "-fPIC", "--offload-arch=gfx950", "-o", tmp] + objs)
        os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build_library(force="--force" in sys.argv, verbose=True))
