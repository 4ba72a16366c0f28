"""Builds libstand.so (HIP, gfx950) in-tree with hipcc."""
import os
import subprocess
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
SOURCES = [os.path.join(HERE, "csrc", f) for f in ("stand_api.hip", "serve_api.hip")]
LIB = os.path.join(HERE, "libstand.so")

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    "-ffp-contract=off",                       # the numeric contract names every fused operation itself
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
]


def build_lib(verbose=False):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    with tempfile.TemporaryDirectory() as d:
        objects = [os.path.join(d, os.path.basename(f) + ".o") for f in SOURCES]
        started = [subprocess.Popen([hipcc] + HIPCC_FLAGS + ["-c", "-o", o, f], stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True)
                   for f, o in zip(SOURCES, objects)]
        results = [(p.communicate(), p.returncode) for p in started]
        if not any(code for _, code in results):
            link = subprocess.run([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB] + objects, capture_output=True, text=True)
            results.append(((link.stdout, link.stderr), link.returncode))
    for (out, err), code in results:
        if verbose or code:
            print(out)
            print(err)
    if any(code for _, code in results):
        raise RuntimeError("hipcc failed building libstand.so")
    return LIB


if __name__ == "__main__":
    print(build_lib(verbose=True))
