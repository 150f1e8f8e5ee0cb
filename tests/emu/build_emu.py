"""Builds the CPU emulation of the library (tests only): the product's host sources plus
emu_lib.cpp, compiled for the host with the clang that ships with ROCm (the kernel header uses
clang vector types), into _build/emu/libalcop_emu.so."""
from __future__ import annotations

import concurrent.futures as cf
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(os.path.dirname(HERE))
CSRC = os.path.join(ROOT, "paper_2210_16691_amd", "csrc")
OUT = os.path.join(ROOT, "_build", "emu")
LIB = os.path.join(OUT, "libalcop_emu.so")
CXX = os.environ.get("ALCOP_HOST_CXX", "/opt/rocm/llvm/bin/clang++")
FLAGS = [os.environ.get("EMU_OPT", "-O1"), "-std=c++17", "-fPIC", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I" + CSRC,
         "-I" + HERE, "-D__launch_bounds__(...)=", "-Wno-psabi", "-Wno-pass-failed"]


def _newest_dep(obj: str) -> float:
    """Newest modification time among the files this object was last compiled from (the compiler's own list; none yet: never
    up to date)."""
    if not os.path.exists(obj + ".d"):
        return float("inf")
    words = open(obj + ".d").read().replace("\\\n", " ").split()
    files = [w for w in words[1:] if not w.endswith(":")]
    return max((os.path.getmtime(f) if os.path.exists(f) else float("inf")) for f in files)


def _compile(job) -> str:
    src, obj, extra = job
    if not os.path.exists(obj) or os.path.getmtime(obj) < _newest_dep(obj):
        subprocess.check_call([CXX] + FLAGS + extra + ["-MD", "-MF", obj + ".d", "-c", src, "-o", obj])
    return obj


def build() -> str:
    os.makedirs(OUT, exist_ok=True)
    emu = os.path.join(HERE, "emu_lib.cpp")
    jobs = [(emu, os.path.join(OUT, "emu_part%d.o" % p), ["-DEMU_PART=%d" % p]) for p in range(8)]
    jobs.append((emu, os.path.join(OUT, "emu_main.o"), ["-DEMU_PART=-1"]))
    for name in ("alcop_api.cpp", "alcop_model.cpp", "alcop_linear.cpp", "alcop_layernorm.cpp", "alcop_grouped.cpp", "alcop_loss.cpp"):
        jobs.append((os.path.join(CSRC, name), os.path.join(OUT, name + ".o"), []))
    lin = os.path.join(HERE, "emu_linear.cpp")
    jobs += [(lin, os.path.join(OUT, "emu_linear%d.o" % p), ["-DEMU_PART=%d" % p]) for p in range(5)]
    jobs.append((os.path.join(HERE, "emu_layernorm.cpp"), os.path.join(OUT, "emu_layernorm.o"), []))
    grouped = os.path.join(HERE, "emu_grouped.cpp")
    jobs += [(grouped, os.path.join(OUT, "emu_grouped%d.o" % p), ["-DEMU_PART=%d" % p]) for p in range(5)]
    jobs += [(os.path.join(HERE, "emu_loss.cpp"), os.path.join(OUT, "emu_loss%d.o" % p), ["-DEMU_PART=%d" % p]) for p in range(3)]
    with cf.ThreadPoolExecutor(max_workers=8) as ex:
        objs = list(ex.map(_compile, jobs))
    if not os.path.exists(LIB) or any(os.path.getmtime(o) > os.path.getmtime(LIB) for o in objs):
        subprocess.check_call([CXX, "-shared", "-o", LIB] + objs +
                              ["-L/opt/rocm/lib", "-lamdhip64", "-Wl,-rpath,/opt/rocm/lib"])
    return LIB


if __name__ == "__main__":
    print(build())
