"""Build librefcache.so in-tree for gfx950 with hipcc.

    python -m paper_2608_21229_amd.build        (or: python paper_2608_21229_amd/build.py)

Every HIP source is compiled with packed-FP32 instruction selection turned
off (-Xclang -target-feature -Xclang -packed-fp32-ops); hipcc's host pass
warns that it does not know that feature, which is harmless.
"""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
import tempfile

if __package__:
    from . import wait_states
else:  # run as a file
    import wait_states

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(PKG, "librefcache.so")
SOURCES = ["layout.cpp", "api.cpp", "attn_fwd.hip", "attn_bwd.hip", "linear.hip", "fp8_cache.hip",
           "rotary.hip", "norm.hip"]
# The attention gradient keeps its output accumulators in accumulation registers
# by its own statements; every other matrix product of it stays in vector ones.
SOURCE_FLAGS = {"attn_bwd.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form=1"]}
# Those statements' wait states depend on what the compiler schedules around them, so
# every build checks the listing of the object that it links.
CHECKED = ["attn_bwd.hip"]
ARCH = "gfx950"


def hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found: install ROCm or set HIPCC")


def compile_command(source: str, out: str, *mode: str) -> list:
    """The hipcc call that compiles one source (mode: -c for an object)."""
    return [hipcc(), f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC", "-Wall", "-Wno-unused-function",
            "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
            # the attention kernels read their by-value arguments at more than
            # 300 places, beyond which LLVM would first copy them to scratch
            "-mllvm", "-instcombine-max-copied-from-constant-users=4096", *SOURCE_FLAGS.get(source, []),
            "-I", INCLUDE, "-I", CSRC, *mode, os.path.join(CSRC, source), "-o", out]


def _finish(cmd, proc, verbose: bool):
    out = proc.communicate()[0]
    errs = "\n".join(l for l in out.splitlines() if "packed-fp32-ops" not in l)
    if verbose:
        print(" ".join(cmd), flush=True)
        if errs.strip():
            print(errs)
    return f"hipcc failed ({proc.returncode}):\n{errs}" if proc.returncode != 0 else None


def _hazards(source: str, objects: str):
    """What is wrong with the listing that was kept beside a checked source's object, or None."""
    name = f"{os.path.splitext(source)[0]}-hip-amdgcn-amd-amdhsa-{ARCH}.s"
    with open(os.path.join(objects, name)) as f:
        products, faults = wait_states.scan(f)
    if faults or not products:
        return (f"{source}: {len(faults)} of {products} accumulator products written as assembly lack wait states in this "
                f"compiler's schedule: {faults[:3]}")
    return None


def build(verbose: bool = False) -> str:
    start = lambda cmd: subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)  # noqa: E731
    with tempfile.TemporaryDirectory() as tmp:
        objs = [os.path.join(tmp, s + ".o") for s in SOURCES]
        cmds = [compile_command(s, o, "-c", *(["--save-temps=obj"] if s in CHECKED else []))
                for s, o in zip(SOURCES, objs)]
        failed = [_finish(c, p, verbose) for c, p in [(c, start(c)) for c in cmds]]
        if not any(failed):
            failed = [_hazards(s, tmp) for s in CHECKED]
        if not any(failed):
            link = [hipcc(), f"--offload-arch={ARCH}", "-fPIC", "-shared", *objs, "-o", LIB + ".tmp"]
            failed = [_finish(link, start(link), verbose)]
    if any(failed):
        raise RuntimeError("\n".join(f for f in failed if f))
    os.replace(LIB + ".tmp", LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
