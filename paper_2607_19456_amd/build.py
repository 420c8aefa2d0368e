"""Build the gfx950 HIP library ``libdecode_attn.so`` in-tree with hipcc: one
object for each of its sources, side by side, then one link.

Used by ``__graft_entry__.build()``; also runnable as
``python -m paper_2607_19456_amd.build``.
"""
from __future__ import annotations

import os
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
SRC = os.path.join(PKG, "csrc", "decode_attn.hip")
PAGED_SRC = os.path.join(PKG, "csrc", "paged_kv.hip")
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(PKG, "libdecode_attn.so")
# The read-ceiling probe the benchmark reports beside the decode (not part of
# the decode).
PROBE_SRC = os.path.join(PKG, "csrc", "hbm_probe.hip")
PROBE_LIB = os.path.join(PKG, "libhbm_probe.so")
# The paged calls' argument handling (a Python extension: host code only).
CALL_SRC = os.path.join(PKG, "csrc", "paged_call.cpp")
CALL_LIB = os.path.join(PKG, "paged_call.so")
ARCH = "gfx950"

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

FLAGS = [
    f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC", "-shared",
    "-Wall", "-Wextra",
    # Keep the compiler from forming packed fp32 instructions.
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # Leave single-lane atomics as they are: the optimizer's wave-wide
    # rewrite reads the result at once, which stalls the load pipeline
    # behind the work counter of the decode kernel.
    "-mllvm", "-amdgpu-atomic-optimizer-strategy=None",
    # Matrix-core results in VGPRs: the decode's accumulators then stay in
    # the registers its softmax rescale works on, instead of being copied
    # between AGPRs and VGPRs around every tile.
    "-mllvm", "-amdgpu-mfma-vgpr-form",
    f"-I{INCLUDE}",
]


def _start(cmd: list, verbose: bool) -> subprocess.Popen:
    if verbose:
        print(" ".join(cmd), flush=True)
    return subprocess.Popen(cmd)


def _finish(jobs: list) -> None:
    failed = [p.args for p in jobs if p.wait() != 0]
    if failed:
        raise subprocess.CalledProcessError(1, failed[0])


def _call_command(out: str) -> list:
    import sysconfig

    import torch
    from torch.utils.cpp_extension import include_paths

    lib = os.path.join(os.path.dirname(torch.__file__), "lib")
    return ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall",
            f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
            *(f"-isystem{p}" for p in include_paths()),
            f"-isystem{sysconfig.get_paths()['include']}", f"-I{INCLUDE}", "-o", out, CALL_SRC,
            f"-L{lib}", "-ltorch_python", "-ltorch_cpu", "-lc10", f"-Wl,-rpath,{lib}"]


def build(verbose: bool = False) -> str:
    """Compile the decode library, the read-ceiling probe and the paged calls'
    argument handling (always; a stale build must never be used).  Returns the
    decode library's path."""
    tag = ".tmp%d" % os.getpid()
    objects = [LIB + tag + ".%d.o" % i for i in range(2)]
    compile_flags = [f for f in FLAGS if f != "-shared"]
    try:
        _finish([_start([HIPCC, *compile_flags, "-c", "-o", obj, src], verbose)
                 for obj, src in zip(objects, (SRC, PAGED_SRC))]
                + [_start([HIPCC, *FLAGS, "-o", PROBE_LIB + tag, PROBE_SRC], verbose),
                   _start(_call_command(CALL_LIB + tag), verbose)])
        _finish([_start([HIPCC, f"--offload-arch={ARCH}", "-shared", "-fPIC", "-o", LIB + tag,
                         *objects], verbose)])
        os.replace(PROBE_LIB + tag, PROBE_LIB)
        os.replace(CALL_LIB + tag, CALL_LIB)
        os.replace(LIB + tag, LIB)
    finally:
        for path in (*objects, LIB + tag, PROBE_LIB + tag, CALL_LIB + tag):
            if os.path.exists(path):
                os.unlink(path)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
