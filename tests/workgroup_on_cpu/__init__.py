"""Kernels compiled for the CPU, a workgroup at a time, with the waves in a chosen order (hip/hip_runtime.h beside this file)."""
import ctypes
import os
import re
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(os.path.dirname(HERE)), "paper_2604_20503_amd", "csrc")
CLANG = "/opt/rocm/llvm/bin/clang++"


def source(name):
    """A kernel's source as it is, but for dynamic LDS, which is the model's, and waits in assembly, which it needs none of."""
    with open(os.path.join(CSRC, name)) as f:
        text = f.read()
    text = re.sub(r"extern __shared__ [^;]*?(\w+)\[\];", r"char* \1 = ::workgroup::dynamic_lds;", text)
    return re.sub(r"asm volatile\([^;]*\);", "", text)


def build(folder, names):
    """A library of the kernels' entry points, and set_wave_order(n): 0 ascending, 1 descending, else shuffled by the seed n."""
    files = {**{n.replace(".hip", ".cpp"): source(n) for n in names},
             "order.cpp": '#include <hip/hip_runtime.h>\nextern "C" void set_wave_order(int n) { workgroup::order = n; }\n'}
    for name, text in files.items():
        with open(os.path.join(folder, name), "w") as f:
            f.write(text)
    lib = os.path.join(folder, "kernels.so")
    subprocess.run([CLANG, "-x", "c++", "-std=c++17", "-O1", "-ffp-contract=on", "-fPIC", "-shared", "-w", "-I", HERE, "-I", CSRC] +
                   [os.path.join(folder, n) for n in files] + ["-o", lib], check=True)
    return ctypes.CDLL(lib)
