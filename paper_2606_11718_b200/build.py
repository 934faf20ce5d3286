"""Build the C-ABI CUDA library (libccl.so) in-tree for sm_100a with nvcc.

``python -m paper_2606_11718_b200.build`` or :func:`build`.  nvcc cross-compiles without a GPU.
"""
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libccl.so")
SOURCES = ["ccl_host.cpp", "ccl_tma.cpp", "ccl_repack.cu", "ccl_traffic.cu", "ccl_gemm.cu", "ccl_gemm_epi.cu", "ccl_bias_grad.cu", "ccl_moe.cu", "ccl_topo.cu"]
NVCC = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")


def _stale():
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + [os.path.join(ROOT, "include", "ccl.h")]
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and not _stale():
        return LIB
    cmd = [NVCC, "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "-shared",
           "-Xcompiler", "-fPIC,-Wall", "-x", "cu", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
           "-cudart", "static", "-o", LIB]
    if verbose:
        cmd += ["-Xptxas", "-v"]
    cmd += [os.path.join(CSRC, s) for s in SOURCES]
    subprocess.run(cmd, check=True)
    return LIB


if __name__ == "__main__":
    import sys
    print(build(force=True, verbose="-v" in sys.argv))
