"""Build libcca.so in-tree with nvcc for sm_100a (no JIT cache, no torch extension machinery)."""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libcca.so")
BIND = os.path.join(HERE, "_bind.so")          # CPython extension: argument marshalling of the 4-bit entry points
SOURCES = ["cca_api.cu", "gemm_simt.cu", "transform.cu", "attn_simt.cu", "tc_kernels.cu", "tc_gemm2.cu", "tc_attn.cu", "tc_attn_bwd.cu", "tc_attn_bwd_fused.cu", "tc_transform.cu", "tc_transform2.cu", "tc_transform_bwd.cu", "decode.cu", "tc_attn256.cu", "transform_unfused.cu", "bwd_unfused.cu", "mla.cu", "qcache.cu", "qlinear.cu", "tc_qlinear.cu"]
NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-Xcompiler", "-fPIC", "--use_fast_math", "-Xptxas", "-v",
]


def _stale() -> bool:
    if not os.path.exists(LIB) or not os.path.exists(BIND):
        return True
    t = min(os.path.getmtime(LIB), os.path.getmtime(BIND))
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC)] + [os.path.join(HERE, "..", "include", "cca.h")]
    return any(os.path.getmtime(p) > t for p in deps)


def _bind_commands(bdir: str):
    """(compile, link) of the extension against this Python and this torch."""
    import sysconfig

    import torch
    root = os.path.dirname(torch.__file__)
    obj = os.path.join(bdir, "bind.o")
    cuda = os.path.join(os.path.dirname(os.path.dirname(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc"))), "include")
    cxx = os.environ.get("CXX", "g++")
    compile_ = [cxx, "-O2", "-std=c++17", "-fPIC", "-fvisibility=hidden", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
                "-I" + os.path.join(root, "include"), "-I" + os.path.join(root, "include", "torch", "csrc", "api", "include"), "-I" + cuda,
                "-I" + sysconfig.get_paths()["include"], "-c", os.path.join(CSRC, "bind.cpp"), "-o", obj]
    link = [cxx, "-shared", "-o", BIND, obj, "-L" + HERE, "-l:libcca.so", "-L" + os.path.join(root, "lib"), "-lc10", "-lc10_cuda",
            "-ltorch_cpu", "-ltorch_cuda", "-ltorch_python", "-Wl,-rpath,$ORIGIN"]
    return compile_, link


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile every .cu into objects (in parallel) and link libcca.so next to this file, then the Python extension over it."""
    if not force and not _stale():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    bdir = os.path.join(HERE, "_build")
    os.makedirs(bdir, exist_ok=True)
    procs = []
    objs = []
    for src in SOURCES:
        obj = os.path.join(bdir, src.replace(".cu", ".o"))
        objs.append(obj)
        cmd = [nvcc, *NVCC_FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    bind_compile, bind_link = _bind_commands(bdir)
    procs.append(("bind.cpp", subprocess.Popen(bind_compile, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    log = []
    for src, p in procs:
        out, _ = p.communicate()
        log.append(f"== {src}\n{out}")
        if p.returncode != 0:
            sys.stderr.write(out)
            raise RuntimeError(f"the compiler failed on {src}")
    with open(os.path.join(bdir, "ptxas.log"), "w") as f:
        f.write("\n".join(log))
    if verbose:
        print("\n".join(log))
    cmd = [nvcc, "-shared", "-o", LIB, *objs, "-lcudart"]
    subprocess.run(cmd, check=True)
    subprocess.run(bind_link, check=True)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
