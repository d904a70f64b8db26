"""Builds the HIP library in-tree:  python -m paper_2510_04212_amd.build

One hipcc invocation per source (gfx950 only).  Four libraries come out:
  libattn_gfx950.so         the attention library (the C ABI of include/attn.h);
  libattn_probe_gfx950.so   measurement aids that only the benchmark loads (csrc/probe.h);
  _autograd.so              the autograd node of attention() (host code, linked against the first);
  _operators.so             plain calls of the rotary positions, the 8-bit cache and the choice among beams (the same).
Packed-fp32 code generation is switched off for all device code.
"""
import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libattn_gfx950.so")
PROBE_LIB = os.path.join(HERE, "libattn_probe_gfx950.so")
NODES = ["autograd", "operators"]              # csrc/NAME.cpp -> _NAME.so
SOURCES = ["api.hip", "fwd.hip", "delta.hip", "bwd.hip", "api_cache.hip", "rope.hip", "cache.hip", "cache_attn.hip", "cache_shared.hip",
           "cache_copy.hip", "beam.hip"]
PROBE_SOURCES = ["probe.hip"]
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-Wno-unused-command-line-argument",
         # the tile loader's inline assembly names m0 as clobbered on purpose (it sets it)
         "-Wno-inline-asm"]
# Per-source additions.  The backward kernels are long straight-line regions of matrix
# instructions with their LDS reads placed by hand; the scheduler's "maximise instruction-level
# parallelism" strategy keeps that order with fewer stalls than the default (occupancy-driven)
# one: measured 2-3 % on the dK/dV kernel at d = 128, nothing lost elsewhere.  The forward is
# faster with the default strategy.
# The forward's matrix instructions write ordinary registers.  By default a kernel that may use more than 256 (d = 256,
# one wave per SIMD) has its accumulators in accumulation registers, which the vector unit reaches by copies only.  The
# scheduler then finds no room for reading ahead from LDS: kernels that need it place their reads themselves
# (kPlacedReads in fwd.hip).  Same bits; us, without the flag -> with it: B2 H8 N2048 d256 causal 87.4 -> 72.6, B4 H8 N1999
# 117 -> 100, B2 H12 N300 21.2 -> 18.5, full B2 H8 N2048 98.9 -> 82.7, N2000 102 -> 85; smaller head sizes as before.
# The backward loses by it (dK/dV B2 H8 N2048 122 -> 131, dQ even).  Attention over the 8-bit cache gains by it at the same head size (2048 queries of 4
# sequences 300 -> 256), others as before.
EXTRA_FLAGS = {"bwd.hip": ["-mllvm", "-amdgpu-sched-strategy=max-ilp"], "fwd.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form=1"],
               "cache_attn.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form=1"], "cache_shared.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form=1"]}


def _node_command(name):
    """One g++ call: csrc/NAME.cpp against torch's C++ interface."""
    import torch
    root = os.path.dirname(torch.__file__)
    return (["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-D__HIP_PLATFORM_AMD__=1", "-DUSE_ROCM=1",
             f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}"]
            + [a for p in (os.path.join(root, "include"), os.path.join(root, "include/torch/csrc/api/include"),
                           sysconfig.get_paths()["include"], "/opt/rocm/include") for a in ("-isystem", p)]
            + [os.path.join(CSRC, name + ".cpp"), "-o", os.path.join(HERE, f"_{name}.so"), "-L" + HERE, "-l:" + os.path.basename(LIB),
               "-Wl,-rpath,$ORIGIN", "-L" + os.path.join(root, "lib"),
               "-ltorch_python", "-ltorch_cpu", "-ltorch_hip", "-lc10_hip", "-lc10"])


def build(verbose=True):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    objdir = os.path.join(HERE, "_build")
    os.makedirs(objdir, exist_ok=True)
    objs = []
    procs = []
    for src in SOURCES + PROBE_SOURCES:
        obj = os.path.join(objdir, src.replace(".hip", ".o"))
        cmd = [hipcc] + FLAGS + EXTRA_FLAGS.get(src, []) + ["-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
        objs.append(obj)
    for src, p in procs:
        out, _ = p.communicate()
        out = "\n".join(l for l in out.splitlines() if "packed-fp32-ops" not in l and l.strip() not in ("", "1 warning generated."))
        if p.returncode != 0:
            raise RuntimeError(f"hipcc failed on {src}:\n{out}")
        if verbose and out.strip():
            print(out)
    for lib, n0, n1 in ((LIB, 0, len(SOURCES)), (PROBE_LIB, len(SOURCES), len(objs))):
        cmd = [hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", lib] + objs[n0:n1]
        if verbose:
            print(" ".join(cmd), flush=True)
        subprocess.run(cmd, check=True)
    procs = []
    for name in NODES:
        cmd = _node_command(name)
        if verbose:
            print(" ".join(cmd), flush=True)
        procs.append((cmd, subprocess.Popen(cmd)))
    for cmd, p in procs:
        if p.wait() != 0:
            raise subprocess.CalledProcessError(p.returncode, cmd)
    return LIB


if __name__ == "__main__":
    build()
    print("built", LIB)
    sys.exit(0)
