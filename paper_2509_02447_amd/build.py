"""Builds libqrm.so (hand-written HIP, gfx950 only) in-tree with hipcc, and the binding's module of host code (_tensors.so) beside it."""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libqrm.so")
MODULE, MODULE_SOURCE = os.path.join(HERE, "_tensors.so"), "tensors.cpp"
OBJ_DIR = os.path.join(HERE, "_build")
SOURCES = ["qrm_api.hip", "extractor.hip", "rs_decode.hip", "tiles.hip", "qrm_noalloc.hip", "qrm_diag.hip", "qrm_plan.hip",
           "qrm_train.hip", "group_norm.hip", "group_norm_f32.hip", "group_norm_bf16.hip",
           "group_norm_f16.hip", "attention.hip", "attention_f32.hip", "attention_bf16.hip", "attention_f16.hip", "adamw.hip",
           "grad_norm.hip", "message_loss.hip"]
HEADERS = ["qrm_internal.h", "qrm_ctx.h", "rs_lane.h", "qrm_train.h", "group_norm.h", "attention.h", os.path.join("..", "..", "include", "qrm.h"),
           os.path.join("..", "..", "include", "qrm_diag.h")]

FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-fvisibility=hidden",
         # packed fp32 arithmetic is kept off for all device code
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-Wno-unused-command-line-argument"]


def hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", "hipcc"):
        if cand and (os.path.isabs(cand) and os.path.exists(cand) or not os.path.isabs(cand)):
            return cand
    return "hipcc"


def stale() -> bool:
    newer = lambda out, deps: not os.path.exists(out) or any(os.path.getmtime(os.path.join(CSRC, d)) > os.path.getmtime(out) for d in deps)
    return newer(LIB, SOURCES + HEADERS) or newer(MODULE, [MODULE_SOURCE])


def build_module() -> str:
    """Compile the CPython module against the torch that is installed."""
    from torch.utils import cpp_extension
    subprocess.check_call([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden"] +
                          ["-I" + p for p in [sysconfig.get_paths()["include"]] + cpp_extension.include_paths()] + [os.path.join(CSRC, MODULE_SOURCE), "-o", MODULE] +
                          ["-L" + p for p in cpp_extension.library_paths()] + ["-ltorch_python", "-ltorch_cpu", "-lc10"])
    return MODULE


def build(force: bool = True, verbose: bool = False) -> str:
    """Compile every HIP source (one hipcc process per file, in parallel) and link paper_2509_02447_amd/libqrm.so."""
    if not force and not stale():
        return LIB
    os.makedirs(OBJ_DIR, exist_ok=True)
    cc = hipcc()

    def compile_one(src: str) -> str:
        obj = os.path.join(OBJ_DIR, src.replace(".hip", ".o"))
        cmd = [cc] + FLAGS + ["-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            cmd.insert(1, "-Rpass-analysis=kernel-resource-usage")
        subprocess.check_call(cmd)
        return obj

    with ThreadPoolExecutor(max_workers=min(8, len(SOURCES))) as pool:
        module = pool.submit(build_module)
        objs = list(pool.map(compile_one, SOURCES))
        module.result()
    subprocess.check_call([cc] + FLAGS + ["-shared"] + objs + ["-o", LIB])
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose="-v" in sys.argv))
