"""Builds libsame.so (HIP kernels for gfx950 + the C ABI + the host graph
compiler) in place, next to this file."""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libsame.so")
SOURCES = ["kernels.hip", "cross_forward.hip", "cross_grad_query.hip", "cross_grad_key.hip", "cross_small.hip",
           "dropout.hip", "qk_norm.hip", "log_probs.hip", "orthogonalise.hip", "ortho_small.hip", "ortho_whole.hip",
           "ortho_columns.hip",
           "api.cpp", "graph.cpp", "operators.cpp", "step.cpp"]
ARCH = os.environ.get("SAME_OFFLOAD_ARCH", "gfx950")

# -packed-fp32-ops: keep the compiler from forming packed fp32 instructions.
# Pairs that the vectoriser forms from scalar code are taken apart again where
# packed fp32 is off, and that has dropped the sign of one of a pair of
# products (negated operand, seen in generated code): nothing is compiled with
# pairs.  Nor may a kernel spill vector registers: a spill at the end of a
# divergent branch has been placed before the lanes come back, and left theirs
# out (seen in generated code).  The remarks name the kernels that do, and a
# library with one is not linked: its answers could be wrong.
HIP_FLAGS = [
    "--offload-arch=" + ARCH, "-O3", "-std=c++17", "-fPIC", "-fno-slp-vectorize",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-Rpass-analysis=kernel-resource-usage",
    "-I" + os.path.join(ROOT, "include"),
]


def spilled(remarks: str) -> list:
    """Kernels with spilled vector registers, from the compiler's resource remarks."""
    names, name = [], "?"
    for line in remarks.splitlines():
        if "Function Name:" in line:
            name = line.split("Function Name:")[1].split()[0]
        elif " VGPRs Spill:" in line and int(line.split("VGPRs Spill:")[1].split()[0]):
            names.append(name)
    return names


def check_remarks(src: str, remarks: str) -> None:
    """Raises where a source's remarks name a kernel that spills, or none at all."""
    if "Function Name:" not in remarks:
        raise RuntimeError("%s: the compiler left no remarks on its kernels' registers" % src)
    if spilled(remarks):
        raise RuntimeError("%s: kernels with spilled vector registers: %s" % (src, ", ".join(spilled(remarks))))


def command(src: str, obj: str) -> list:
    """The compiler's call for one source."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if src.endswith(".cpp"):
        return [hipcc, "-O3", "-std=c++17", "-fPIC", "-I" + os.path.join(ROOT, "include"),
                "-c", os.path.join(CSRC, src), "-o", obj]
    return [hipcc] + HIP_FLAGS + ["-c", os.path.join(CSRC, src), "-o", obj]


def build(verbose: bool = False) -> str:
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    objdir = os.path.join(HERE, "_build")
    os.makedirs(objdir, exist_ok=True)
    objs, jobs = [], []
    for src in SOURCES:
        obj = os.path.join(objdir, src + ".o")
        cmd = command(src, obj)
        if verbose:
            print(" ".join(cmd), flush=True)
        log = open(obj + ".log", "w") if src.endswith(".hip") else None
        jobs.append((src, cmd, subprocess.Popen(cmd, stderr=log), log))
        objs.append(obj)
    failed = [(cmd, log) for _, cmd, job, log in jobs if job.wait() != 0]
    remarks = {}
    for src, _, _, log in jobs:
        if log:
            log.close()
            with open(log.name) as f:
                remarks[src] = f.read()
    if failed:
        cmd, log = failed[0]
        if log:
            with open(log.name) as f:
                sys.stderr.write(f.read())
        raise subprocess.CalledProcessError(1, cmd)
    for src, text in remarks.items():
        check_remarks(src, text)
    tmp = LIB + ".tmp%d" % os.getpid()
    cmd = [hipcc, "--offload-arch=" + ARCH, "-shared", "-fPIC", "-o", tmp] + objs
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.check_call(cmd)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    build(verbose="-v" in sys.argv)
    print(LIB)
