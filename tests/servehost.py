"""Plain host code of the operators around a verification, compiled with the host compiler: `build` gives a library of the
functions of a C++ source that includes the headers of csrc/."""
import ctypes as C
import os
import subprocess
import tempfile

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2506_04708_amd", "csrc")


def build(source, functions):
    """functions: name -> (argument types, result type)."""
    with tempfile.TemporaryDirectory() as d:
        src, so = os.path.join(d, "host.cpp"), os.path.join(d, "host.so")
        open(src, "w").write(source)
        subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", CSRC, "-o", so, src], check=True)
        lib = C.CDLL(so)
    for name, (args, res) in functions.items():
        f = getattr(lib, name)
        f.argtypes, f.restype = args, res
    return lib
