"""Builds libsali.so (the HIP kernels + C ABI) in-tree with hipcc for gfx950.

Usage: python -m paper_2602_14236_amd.build   (or call build()).
"""
from __future__ import annotations

import os
import re
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
OUT = os.path.join(HERE, "libsali.so")

COMMON = [
    "--offload-arch=gfx950", "-O3", "-fPIC", "-std=c++17", "-Wall", "-Wno-unused-function",
    # packed fp32 instructions are kept out of the generated code on this target
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # the first scalar arguments of a kernel come in registers; what depends on them need not wait for a load
    "-mllvm", "-amdgpu-kernarg-preload-count=16",
    "-I", os.path.join(ROOT, "include"), "-I", CSRC,
]

# per-file extra flags: the quantiser must not fuse multiply-adds (codes are defined by
# single fp32 operations); the flow and attention kernels may.
SOURCES = {
    "api.hip": [],
    "kv_kernels.hip": ["-ffp-contract=off"],
    "attn_kernels.hip": ["-ffp-contract=fast"],
    "saliency_kernels.hip": [],
    "flow_kernels.hip": ["-ffp-contract=fast"],
    "pages_api.hip": [],
    "pages_kernels.hip": ["-ffp-contract=off"],
    "pages_attn_fp16.hip": ["-ffp-contract=fast"],
    "pages_attn_bf16.hip": ["-ffp-contract=fast"],
}

# Kernels whose registers have to suffice.  Where a vector register was spilled in one of them, the compiler put the store at the head of a block ahead of
# the instruction that brings the masked lanes back, and waves reloaded what they had never stored; the build refuses such code.
NO_SPILLS = ("pages_attn_fp16.hip", "pages_attn_bf16.hip")
REPORT = ["-Rpass-analysis=kernel-resource-usage"]


def spilled(report: str):
    """Names of the kernels that spill vector registers, from the compiler's report."""
    name, bad = "?", []
    for line in report.splitlines():
        m = re.search(r"remark: .*?(Function Name|VGPRs Spill): (\S+)", line)
        if m and m.group(1) == "Function Name":
            name = m.group(2)
        elif m and m.group(2) != "0":
            bad.append(name)
    return bad


def build(verbose: bool = True) -> str:
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    bdir = os.path.join(HERE, "_build")
    os.makedirs(bdir, exist_ok=True)
    objs = []
    procs = []
    for src, extra in SOURCES.items():
        obj = os.path.join(bdir, src.replace(".hip", ".o"))
        if src in NO_SPILLS:
            extra = [*extra, *REPORT]
        cmd = [hipcc, *COMMON, *extra, "-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
        objs.append(obj)
    failed = False
    for src, p in procs:
        out, _ = p.communicate()
        if src in NO_SPILLS:
            bad = spilled(out)
            if bad:
                print(f"{src}: vector registers are spilled in {', '.join(bad)}", file=sys.stderr)
                failed = True
            if p.returncode == 0:
                out = ""                        # the report
        out = "\n".join(l for l in out.splitlines() if "packed-fp32-ops" not in l and "warning generated" not in l)
        if out.strip() and verbose:
            print(out)
        if p.returncode != 0:
            print(f"hipcc failed on {src}", file=sys.stderr)
            failed = True
    if failed:
        raise RuntimeError("libsali build failed")
    cmd = [hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", *objs, "-o", OUT]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)
    return OUT


if __name__ == "__main__":
    build()
