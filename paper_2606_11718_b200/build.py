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
    """Compiles the sources side by side (one object each) and links them into libccl.so."""
    if not force and not _stale():
        return LIB
    objdir = os.path.join(HERE, "build")
    os.makedirs(objdir, exist_ok=True)
    flags = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "-Xcompiler", "-fPIC,-Wall", "-x", "cu",
             "-I", os.path.join(ROOT, "include"), "-I", CSRC]
    if verbose:
        flags += ["-Xptxas", "-v"]
    headers = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".h", ".cuh"))] + [os.path.join(ROOT, "include", "ccl.h")]
    newest = max(os.path.getmtime(h) for h in headers)
    objects, running = [], []
    for src in SOURCES:
        path, obj = os.path.join(CSRC, src), os.path.join(objdir, src + ".o")
        objects.append(obj)
        if force or not os.path.exists(obj) or os.path.getmtime(obj) < max(newest, os.path.getmtime(path)):
            cmd = [NVCC] + flags + ["-c", path, "-o", obj]
            running.append((cmd, obj, subprocess.Popen(cmd)))
    failed = [(p.returncode, cmd, obj) for cmd, obj, p in running if p.wait()]
    for rc, cmd, obj in failed:
        if os.path.exists(obj):
            os.remove(obj)
    if failed:
        raise subprocess.CalledProcessError(failed[0][0], failed[0][1])
    subprocess.run([NVCC, "-gencode", "arch=compute_100a,code=sm_100a", "-shared", "-cudart", "static", "-o", LIB] + objects, check=True)
    return LIB


if __name__ == "__main__":
    import sys
    print(build(force=True, verbose="-v" in sys.argv))
