"""Build libcca.so in-tree with nvcc for sm_100a (no JIT cache, no torch extension machinery)."""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libcca.so")
HEADER = os.path.join(HERE, "..", "include", "cca.h")
BIND = os.path.join(HERE, "_bind.so")          # CPython extension: argument marshalling of the 4-bit entry points
SOURCES = ["cca_api.cu", "gemm_simt.cu", "transform.cu", "attn_simt.cu", "tc_kernels.cu", "tc_gemm2.cu", "tc_attn.cu", "tc_attn_bwd.cu", "tc_attn_bwd_fused.cu", "tc_transform.cu", "tc_transform2.cu", "tc_transform_bwd.cu", "decode.cu", "tc_attn256.cu", "transform_unfused.cu", "bwd_unfused.cu", "mla.cu", "qcache.cu", "qlinear.cu", "tc_qlinear.cu"]
NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-Xcompiler", "-fPIC", "--use_fast_math", "-Xptxas", "-v",
]


def _older(path: str, deps) -> bool:
    return not os.path.exists(path) or any(os.path.getmtime(d) > os.path.getmtime(path) for d in deps)


def _lib_stale() -> bool:
    return _older(LIB, [os.path.join(CSRC, f) for f in os.listdir(CSRC) if not f.endswith(".cpp")] + [HEADER])


def _built_for() -> str:
    """The Python and the torch that the extension is compiled against; it carries this text."""
    import sysconfig

    import torch
    return f"built for {sysconfig.get_config_var('SOABI')}, torch {torch.__version__}"


def bind_fits() -> bool:
    """Whether there is an extension and it was compiled against this Python and this torch."""
    if not os.path.exists(BIND):
        return False
    with open(BIND, "rb") as f:
        return _built_for().encode() + b"\0" in f.read()


def _bind_stale() -> bool:
    return _older(BIND, [os.path.join(CSRC, "bind.cpp"), HEADER]) or not bind_fits()


def _stale() -> bool:
    return _lib_stale() or _bind_stale()


def _bind_commands(bdir: str):
    """(compile, link) of the extension against this Python and this torch."""
    import sysconfig

    import torch
    root = os.path.dirname(torch.__file__)
    obj = os.path.join(bdir, "bind.o")
    cuda = os.path.join(os.path.dirname(os.path.dirname(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc"))), "include")
    cxx = os.environ.get("CXX", "g++")
    compile_ = [cxx, "-O2", "-std=c++17", "-fPIC", "-fvisibility=hidden", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
                f'-DCCA_BUILT_FOR="{_built_for()}"',
                "-I" + os.path.join(root, "include"), "-I" + os.path.join(root, "include", "torch", "csrc", "api", "include"), "-I" + cuda,
                "-I" + sysconfig.get_paths()["include"], "-c", os.path.join(CSRC, "bind.cpp"), "-o", obj]
    link = [cxx, "-shared", "-o", BIND, obj, "-L" + HERE, "-l:libcca.so", "-L" + os.path.join(root, "lib"), "-lc10", "-lc10_cuda",
            "-ltorch_cpu", "-ltorch_cuda", "-ltorch_python", "-Wl,-rpath,$ORIGIN"]
    return compile_, link


def _finish(src: str, p, log) -> None:
    out, _ = p.communicate()
    log.append(f"== {src}\n{out}")
    if p.returncode != 0:
        sys.stderr.write(out)
        raise RuntimeError(f"the compiler failed on {src}")


def _start(cmd):
    return subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)


def build_library(force: bool = False, verbose: bool = False) -> str:
    """Compile every .cu into objects (in parallel) and link libcca.so next to this file."""
    if not force and not _lib_stale():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    bdir = os.path.join(HERE, "_build")
    os.makedirs(bdir, exist_ok=True)
    procs = []
    objs = []
    for src in SOURCES:
        obj = os.path.join(bdir, src.replace(".cu", ".o"))
        objs.append(obj)
        procs.append((src, _start([nvcc, *NVCC_FLAGS, "-c", os.path.join(CSRC, src), "-o", obj])))
    log = []
    for src, p in procs:
        _finish(src, p, log)
    with open(os.path.join(bdir, "ptxas.log"), "w") as f:
        f.write("\n".join(log))
    if verbose:
        print("\n".join(log))
    subprocess.run([nvcc, "-shared", "-o", LIB, *objs, "-lcudart"], check=True)
    return LIB


def build_bind(force: bool = False) -> str:
    """Compile the Python extension and link it over libcca.so, which has to be there."""
    if not force and not _bind_stale():
        return BIND
    bdir = os.path.join(HERE, "_build")
    os.makedirs(bdir, exist_ok=True)
    compile_, link = _bind_commands(bdir)
    _finish("bind.cpp", _start(compile_), [])
    subprocess.run(link, check=True)
    return BIND


def build(force: bool = False, verbose: bool = False) -> str:
    """The library, then the Python extension over it."""
    build_library(force, verbose)
    build_bind(force)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
