"""Host functions of the library's headers, compiled by nvcc into a shared object for a test that has no GPU."""
import ctypes
import os
import subprocess

from paper_2506_07366_b200 import build


def compiled(folder, source: str):
    """The shared object of `source`, CUDA C++ that may include csrc and include headers."""
    path = os.path.join(str(folder), "host_code")
    with open(path + ".cu", "w") as f:
        f.write(source)
    proc = subprocess.run([build._nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-shared", "-Xcompiler", "-fPIC",
                           "-I", os.path.join(build.ROOT, "include"), "-I", build.CSRC, path + ".cu", "-o", path + ".so"],
                          capture_output=True, text=True)
    assert proc.returncode == 0, proc.stderr
    return ctypes.CDLL(path + ".so")
