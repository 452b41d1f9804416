"""The library's host code on a CUDA runtime of the host (fake_cudart.cpp): its
objects linked with that in place of CUDA's.  No GPU is needed, and none used."""

import ctypes
import os
import subprocess

from paper_2606_14782_gb300 import bacon, build

HERE = os.path.dirname(os.path.abspath(__file__))


def library(folder):
    """libbacon of the present sources with the runtime of the host, bound like
    bacon.load() binds it."""
    build.build()
    sources = [p for p in build.inputs() if p.endswith(".cu")]
    objects = [os.path.join(build.BUILD, os.path.basename(p)[:-3] + ".o") for p in sources]
    newest = max(os.path.getmtime(p) for p in build.inputs())
    if not all(os.path.exists(o) and os.path.getmtime(o) >= newest for o in objects):
        build.build(force=True)
    fake, lib = os.path.join(folder, "fake.o"), os.path.join(folder, "libfake.so")
    cc = build.nvcc()
    subprocess.run([cc, "-c", os.path.join(HERE, "fake_cudart.cpp"), "-o", fake, "-std=c++17",
                    "-Xcompiler", "-fPIC"], check=True)
    # its own symbols first, whatever the process has loaded
    subprocess.run([cc, "-shared", "-o", lib, fake] + objects
                   + ["-cudart", "none", "-Xcompiler", "-fPIC", "-Xlinker", "-Bsymbolic"],
                   check=True)
    kept = bacon.LIB_PATH, bacon._lib
    bacon.LIB_PATH, bacon._lib = lib, None
    try:
        bound = bacon.load()
    finally:
        bacon.LIB_PATH, bacon._lib = kept
    bound.fake_last_allocation.restype = ctypes.c_void_p
    bound.fake_last_allocation.argtypes = [ctypes.POINTER(ctypes.c_size_t)]
    bound.fake_allocation_of.restype = ctypes.c_void_p
    bound.fake_allocation_of.argtypes = [ctypes.c_size_t]
    bound.fake_device_work.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int]
    bound.fake_device_work.restype = None
    return bound
