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
NARROW = 1 << 14  # lanes of a launch at most in the library whose launches are in many turns
CLANG = "/opt/rocm/llvm/bin/clang++"


def _run(cmd):
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("emulation build failed: %s\n%s" % (" ".join(cmd[-3:]), res.stderr[-4000:]))


def _compile(src, flags=()):
    obj = os.path.join(OBJ, os.path.basename(src) + (".narrow.o" if flags else ".o"))
    _run([CLANG, "-O2", "-std=c++17", "-fPIC", "-w", "-x", "c++", "-c", "-I", os.path.join(HERE, "local"), "-I", os.path.join(HERE, "include"),
          *flags, src, "-o", obj])
    return obj


def build(narrow=False):
    out = OUT.replace(".so", "_narrow.so") if narrow else OUT
    flags = ["-DHAFLO_LOCAL_LANES=%d" % NARROW, "-DHIPEMU_LANES=%d" % NARROW] if narrow else []
    srcs = sorted(glob.glob(os.path.join(CSRC, "local_*.hip"))) + [os.path.join(HERE, "hipemu.cpp")]
    used = srcs + [os.path.join(CSRC, "local_common.hpp"), os.path.join(HERE, "include", "hip", "hip_runtime.h"),
                   os.path.join(HERE, "local", "hip", "hip_runtime.h"), os.path.join(ROOT, "include", "haflo_local.h"),
                   os.path.abspath(__file__)]
    if os.path.exists(out) and os.path.getmtime(out) >= max(os.path.getmtime(p) for p in used):
        return out
    os.makedirs(OBJ, exist_ok=True)
    with ThreadPoolExecutor(max_workers=4) as pool:
        objs = list(pool.map(lambda src: _compile(src, flags), srcs))
    _run([CLANG, "-shared", "-fPIC"] + objs + ["-o", out])
    return out


if __name__ == "__main__":
    print(build())
