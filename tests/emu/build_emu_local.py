"""Build the CPU-emulated library of a party's local operators: their own sources compiled for the host by clang against
tests/emu/local, with the scheduler behind the stand-in for the HIP runtime."""
import glob
import os
import subprocess
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(os.path.dirname(HERE))
CSRC = os.path.join(ROOT, "paper_2107_13797_amd", "csrc")
OUT = os.path.join(HERE, "libhaflo_emu_local.so")
OBJ = os.path.join(HERE, "_build", "local")
CLANG = "/opt/rocm/llvm/bin/clang++"


def _run(cmd):
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("emulation build failed: %s\n%s" % (" ".join(cmd[-3:]), res.stderr[-4000:]))


def _compile(src):
    obj = os.path.join(OBJ, os.path.basename(src) + ".o")
    _run([CLANG, "-O2", "-std=c++17", "-fPIC", "-w", "-x", "c++", "-c", "-I", os.path.join(HERE, "local"), "-I", os.path.join(HERE, "include"),
          src, "-o", obj])
    return obj


def build():
    srcs = sorted(glob.glob(os.path.join(CSRC, "local_*.hip"))) + [os.path.join(HERE, "hipemu.cpp")]
    used = srcs + [os.path.join(CSRC, "local_common.hpp"), os.path.join(HERE, "include", "hip", "hip_runtime.h"),
                   os.path.join(HERE, "local", "hip", "hip_runtime.h"), os.path.join(ROOT, "include", "haflo_local.h"),
                   os.path.abspath(__file__)]
    if os.path.exists(OUT) and os.path.getmtime(OUT) >= max(os.path.getmtime(p) for p in used):
        return OUT
    os.makedirs(OBJ, exist_ok=True)
    with ThreadPoolExecutor(max_workers=4) as pool:
        objs = list(pool.map(_compile, srcs))
    _run([CLANG, "-shared", "-fPIC"] + objs + ["-o", OUT])
    return OUT


if __name__ == "__main__":
    print(build())
