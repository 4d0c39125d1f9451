"""Build libentro.so in-tree: g++ for the host part, hipcc (gfx950) for the kernels."""
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(HERE, "libentro.so")
BUILD = os.path.join(HERE, "_build")

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
# -packed-fp32-ops off: the compiler must not form packed fp32 instructions
DEVICE_FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Xclang", "-target-feature",
                "-Xclang", "-packed-fp32-ops", "-Wno-unused-command-line-argument"]


DEVICE_SOURCES = ["entro_device", "entro_compress", "entro_cache", "entro_attend"]


def sources():
    return [os.path.join(CSRC, "entro_host.cpp"), os.path.join(CSRC, "entro_cache.h"), os.path.join(INCLUDE, "entro.h"),
            *(os.path.join(CSRC, name + ".hip") for name in DEVICE_SOURCES)]


def up_to_date() -> bool:
    return os.path.exists(LIB) and all(os.path.getmtime(LIB) >= os.path.getmtime(s) for s in sources())


def build(force: bool = True, verbose: bool = False) -> str:
    if not force and up_to_date():
        return LIB
    os.makedirs(BUILD, exist_ok=True)
    objects = [os.path.join(BUILD, name + ".o") for name in ["entro_host", *DEVICE_SOURCES]]
    cmds = [["g++", "-O3", "-std=c++17", "-fPIC", "-ffp-contract=off", "-Wall", "-Wextra", "-pthread",
             "-I", INCLUDE, "-c", os.path.join(CSRC, "entro_host.cpp"), "-o", objects[0]]]
    cmds += [[HIPCC, *DEVICE_FLAGS, "-I", INCLUDE, "-c", os.path.join(CSRC, name + ".hip"), "-o", o]
             for name, o in zip(DEVICE_SOURCES, objects[1:])]
    link = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB, *objects, "-pthread"]
    # the sources compile side by side
    running = []
    for c in cmds:
        if verbose:
            print(" ".join(c), flush=True)
        running.append((c, subprocess.Popen(c)))
    failed = [(c, p.returncode) for c, p in running if p.wait() != 0]
    if failed:
        raise subprocess.CalledProcessError(failed[0][1], failed[0][0])
    if verbose:
        print(" ".join(link), flush=True)
    subprocess.check_call(link)
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose="-v" in sys.argv))
