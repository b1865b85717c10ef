"""Build libellm.so (HIP, gfx950) in-tree with hipcc, and _calls, the native part of the Python binding, with g++."""
from __future__ import annotations

import os
import subprocess
import sysconfig
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libellm.so")
# (named for the interpreter it is built for: another one does not load it)
CALLS = os.path.join(HERE, "_calls" + sysconfig.get_config_var("EXT_SUFFIX"))
CALLS_SOURCE = os.path.join(CSRC, "python_calls.cpp")
SOURCES = ["pool_core.cpp", "ellm_api.cpp", "kernels.hip", "kernels_fp4.hip", "kernels_tokens.hip"]
HEADERS = ["pool_core.hpp", "kernels.hpp", "device.hpp", "fp4.hpp", "fp4_walk.hpp", "divide.hpp", "map_queue.hpp", os.path.join(ROOT, "include", "ellm.h")]

# packed-fp32 instructions are switched off for all device code of this library
DEVICE_FLAGS = ["-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]


def needs_build() -> bool:
    if not os.path.exists(LIB) or not os.path.exists(CALLS) or os.path.getmtime(CALLS_SOURCE) > os.path.getmtime(CALLS):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, s) for s in SOURCES] + [h if os.path.isabs(h) else os.path.join(CSRC, h) for h in HEADERS]
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = True, verbose: bool = False) -> str:
    if not force and not needs_build():
        return LIB
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    import numpy
    calls = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", "-I", sysconfig.get_paths()["include"],
             "-I", numpy.get_include(), CALLS_SOURCE, "-o", CALLS]
    # every source by a compiler of its own, all at once: most of the time goes into the two files of kernels
    with tempfile.TemporaryDirectory() as tmp:
        objects = [os.path.join(tmp, s + ".o") for s in SOURCES]
        compiles = [[hipcc, "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Wall", "-Wno-unused-result",
                     *(DEVICE_FLAGS if s.endswith(".hip") else []), "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-c",
                     os.path.join(CSRC, s), "-o", o] for s, o in zip(SOURCES, objects)] + [calls]
        link = [hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", *objects, "-o", LIB]
        if verbose:
            print("\n".join(" ".join(c) for c in [*compiles, link]))
        running = [(c, subprocess.Popen(c)) for c in compiles]
        status = [(c, p.wait()) for c, p in running]      # (all of them, also where one has failed)
        for c, rc in status:
            if rc:
                raise subprocess.CalledProcessError(rc, c)
        subprocess.run(link, check=True)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
