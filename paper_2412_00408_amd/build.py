"""Build libquake.so for gfx950 with hipcc (in-tree, next to this file).

    python -m paper_2412_00408_amd.build

Every source is compiled for gfx950 only, with fp contraction off (every
fused multiply-add of the method is an explicit fma), packed-fp32 VALU ops
disabled, denormals kept, then linked into one shared library.
"""
from __future__ import annotations

import glob
import os
import re
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD_DIR = os.path.join(ROOT, "_build")
LIB = os.path.join(HERE, "libquake.so")
C_CLIENT_SRC = os.path.join(ROOT, "tests", "c", "abi_smoke.c")
C_CLIENT = os.path.join(ROOT, "tests", "c", "abi_smoke")
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")

SOURCES = ["elementwise.hip", "softmax.hip", "native16.hip", "gemm.hip", "attention.hip",
           "window.hip", "sample.hip", "distill.hip", "ceiling.hip", "abi.cpp"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
ARCH = "gfx950"
FLAGS = [
    "--offload-arch=" + ARCH, "-O3", "-std=c++17", "-fPIC", "-ffp-contract=off",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-command-line-argument", "-I", INCLUDE, "-I", CSRC,
]


# Matrix-core accumulators in ordinary VGPRs: the attention kernels feed them
# straight to VALU work, which cannot read the accumulation registers.
EXTRA_FLAGS = {"attention.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"],
               "window.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"]}


SHIFT64 = re.compile(r"\bv_(?:lshlrev_b64|lshrrev_b64|ashrrev_i64)\S* v\[\d+:\d+\], v(\d+),")


def shifts_by_the_last_register(assembly: str) -> list[str]:
    """Kernels with a 64-bit shift whose amount lies in the last vector register of
    their allocation (which is in eights). The GPU reads the amount as a pair, takes
    the missing half's place from v0 and shifts by that; the compiler does not avoid
    it."""
    bad = []
    for name, regs in re.findall(r"\.amdhsa_kernel (\S+).*?\.amdhsa_next_free_vgpr (\d+)", assembly, re.S):
        at = assembly.index("\n%s:" % name)
        last = (int(regs) + 7) // 8 * 8 - 1
        if any(int(a) == last for a in SHIFT64.findall(assembly[at:assembly.index(".Lfunc_end", at)])):
            bad.append(name)
    return bad


def _compile(src: str) -> str:
    name = os.path.basename(src)
    obj = os.path.join(BUILD_DIR, name + ".o")
    lang = ["-x", "hip"] if src.endswith(".cpp") else EXTRA_FLAGS.get(src, [])
    with tempfile.TemporaryDirectory(dir=BUILD_DIR, prefix=name + ".") as temps:
        out = os.path.join(temps, name + ".o")           # and the compiled code as text beside it
        r = subprocess.run([HIPCC, *lang, *FLAGS, "-c", os.path.join(CSRC, src), "-save-temps=obj", "-o", out],
                           capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError("hipcc failed for %s:\n%s\n%s" % (src, r.stdout, r.stderr))
        (text,) = glob.glob(os.path.join(temps, "*amdgcn*%s.s" % ARCH))
        with open(text) as f:
            bad = shifts_by_the_last_register(f.read())
        if bad:
            raise RuntimeError("%s: a 64-bit shift by the last register, which the GPU gets wrong, in %s"
                               % (src, ", ".join(bad)))
        os.replace(out, obj)
    return obj


def build(verbose: bool = False) -> str:
    os.makedirs(BUILD_DIR, exist_ok=True)
    with ThreadPoolExecutor(min(len(SOURCES), os.cpu_count() or 1)) as ex:
        objs = list(ex.map(_compile, SOURCES))
    tmp = LIB + ".tmp%d" % os.getpid()
    cmd = [HIPCC, "--offload-arch=" + ARCH, "-shared", "-fPIC", "-o", tmp, *objs]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed:\n%s\n%s" % (r.stdout, r.stderr))
    os.replace(tmp, LIB)
    if verbose:
        print("built", LIB)
    return LIB


def build_c_client(verbose: bool = False) -> str:
    """Compile the plain-C client of the ABI (gcc, include/quake.h and the HIP
    runtime only) that checks the library from C, without Python or torch."""
    cmd = ["gcc", "-std=c11", "-O2", "-Wall", "-D__HIP_PLATFORM_AMD__", "-I", INCLUDE,
           "-I", os.path.join(ROCM, "include"), C_CLIENT_SRC, "-o", C_CLIENT + ".tmp",
           "-L", HERE, "-lquake", "-L", os.path.join(ROCM, "lib"), "-lamdhip64", "-lm",
           "-Wl,-rpath,$ORIGIN/../../paper_2412_00408_amd",
           "-Wl,-rpath," + os.path.join(ROCM, "lib")]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("gcc failed for the C client:\n%s\n%s" % (r.stdout, r.stderr))
    os.replace(C_CLIENT + ".tmp", C_CLIENT)
    if verbose:
        print("built", C_CLIENT)
    return C_CLIENT


if __name__ == "__main__":
    build(verbose=True)
    build_c_client(verbose=True)
    sys.exit(0)
