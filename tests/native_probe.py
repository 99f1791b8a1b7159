"""Compiles small programs against the library's device headers, for tests of parts that no entry point reaches by itself."""
import ctypes as C
import os
import subprocess

from paper_2605_29860_b200 import build


def compile_probe(source: str, folder) -> C.CDLL:
    src, out = os.path.join(str(folder), "probe.cu"), os.path.join(str(folder), "probe.so")
    with open(src, "w") as f:
        f.write(source)
    subprocess.run([build._nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-O1", "-std=c++17", "-w", "-Xcompiler", "-fPIC",
                    "-shared", "-I", build._INCLUDE, "-I", build._CSRC, "-o", out, src], check=True)
    return C.CDLL(out)
