"""Build libpuro.so (HIP for gfx950) in-tree with hipcc.

Each source compiles to an object in parallel (the GEMM kernel once per
variant); the objects link into
``paper_2608_27370_amd/libpuro.so``. Packed-FP32 instruction selection is
disabled for all device code.
"""

import concurrent.futures
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libpuro.so")
# (source, object name, extra flags): the GEMM kernel is compiled once per
# operand-format pair and scale kind, so that its instantiations build in parallel
GEMM_VARIANTS = [(fa, fb, g) for fa in (0, 1) for fb in (0, 1) for g in (0, 1)] + [(2, 2, 0), (3, 3, 0)]   # + BF16, int8
SOURCES = [("quant.hip", "quant", []), ("qk_quant.hip", "qk_quant", []),
           ("qk_norm_rope.hip", "qk_norm_rope", []), ("gemm.hip", "gemm", []), ("lm_head.hip", "lm_head", []),
           ("lm_distill.hip", "lm_distill", []), ("int8.hip", "int8", []), ("verify.hip", "verify", []),
           ("transpose.hip", "transpose", []), ("muonh.hip", "muonh", []), ("api.cpp", "api", [])] + [
    ("gemm_kernel.hip", "gemm_kernel_%d%d%d" % v, ["-DPURO_FA=%d" % v[0], "-DPURO_FB=%d" % v[1], "-DPURO_GROUPED=%d" % v[2]])
    for v in GEMM_VARIANTS]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Wall",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-I", INCLUDE, "-I", CSRC]


def _compile(entry):
    src, name, extra = entry
    obj = os.path.join(BUILD, name + ".o")
    cmd = [HIPCC] + FLAGS + extra + ["-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    # the host pass does not know the device-only target feature; that note is harmless
    err = "\n".join(l for l in r.stderr.splitlines() if "packed-fp32-ops" not in l)
    if r.returncode != 0:
        raise RuntimeError("hipcc failed for %s:\n%s" % (src, err))
    return obj


def build(verbose=False):
    os.makedirs(BUILD, exist_ok=True)
    with concurrent.futures.ThreadPoolExecutor(min(len(SOURCES), os.cpu_count() or 1)) as ex:
        objs = list(ex.map(_compile, SOURCES))
    tmp = LIB + ".tmp%d" % os.getpid()
    cmd = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", tmp] + objs
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed:\n" + r.stderr)
    os.replace(tmp, LIB)
    if verbose:
        print("built", LIB)
    return LIB


if __name__ == "__main__":
    build(verbose=True)
    sys.exit(0)
