"""Builds libgdn_tailreplay.so (HIP, gfx950) in-tree.

``python -m paper_2608_30310_amd.build``.  Cross-compiles on a machine without
a GPU; the shared library lands next to this file.
"""
from __future__ import annotations

import os
import shutil
import subprocess
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB_NAME = "libgdn_tailreplay.so"
LIB_PATH = os.path.join(HERE, LIB_NAME)
SOURCES = ["gdn_plan.cpp", "gdn_layer_plan.cpp", "gdn_gemm.cpp", "gdn_api.hip", "gdn_block.hip", "gdn_conv.hip",
           "gdn_ssm.hip", "gdn_linear.hip", "gdn_lora.hip", "gdn_attn_plan.cpp", "gdn_pages.hip", "gdn_attn.hip"]
ROCM_LIB = "/opt/rocm/lib"
ARCH = "gfx950"


def hipcc() -> str:
    path = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(path):
        raise RuntimeError("hipcc not found: the HIP toolchain is required")
    return path


def build(verbose: bool = False) -> str:
    tmp = LIB_PATH + ".tmp"
    flags = [f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC",
             # packed fp32 instructions stay off on this target
             "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
             # MFMA results in ordinary VGPRs: the scan feeds them to VALU work
             # every step, and accumulator-register copies would serialise it
             "-mllvm", "-amdgpu-mfma-vgpr-form",
             # (a clobber of M0, which the loads into LDS set, is reported for each of them)
             "-Wno-inline-asm",
             "-Wall", "-I", INCLUDE, "-I", CSRC]
    noise = "is not a recognized feature for this target"

    def run(cmd):
        res = subprocess.run(cmd, capture_output=True, text=True)
        msgs = [l for l in (res.stdout + res.stderr).splitlines() if noise not in l]
        if res.returncode != 0:
            raise RuntimeError("hipcc failed:\n" + " ".join(cmd) + "\n" + "\n".join(msgs))
        return msgs

    # the sources side by side, as many as there are CPUs for (about 1 GiB each)
    with tempfile.TemporaryDirectory() as objs:
        pairs = [(os.path.join(CSRC, s), os.path.join(objs, s + ".o")) for s in SOURCES]
        cmds = [[hipcc(), *flags, "-c", "-o", obj, src] for src, obj in pairs]
        # the layer block's projections run through hipBLASLt
        link = [hipcc(), f"--offload-arch={ARCH}", "-shared", "-fPIC", "-o", tmp, *(obj for _, obj in pairs),
                "-L", ROCM_LIB, "-Wl,-rpath," + ROCM_LIB, "-lhipblaslt"]
        if verbose:
            print("\n".join(" ".join(c) for c in cmds + [link]), flush=True)
        with ThreadPoolExecutor(max_workers=max(1, min(8, os.cpu_count() or 1))) as pool:
            msgs = [m for out in pool.map(run, cmds) for m in out]
        msgs += run(link)
    if verbose and msgs:
        print("\n".join(msgs))
    os.replace(tmp, LIB_PATH)
    return LIB_PATH


if __name__ == "__main__":
    print(build(verbose=True))
