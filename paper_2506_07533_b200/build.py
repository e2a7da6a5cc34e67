"""Builds libmoqae.so in-tree with nvcc for sm_100a (cross-compiles without a GPU)."""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libmoqae.so")
MARSHAL = os.path.join(HERE, "_marshal.so")      # Python module: tensors in, C ABI structs out
SOURCES = ["api.cu", "route.cu", "quantize.cu", "decode.cu", "decode_mma.cu", "decode_static.cu", "prefill.cu", "project.cu",
           "paged_api.cu", "paged_append.cu", "paged_decode.cu", "paged_prefill.cu", "paged_plan.cu", "paged4_append.cu", "paged4_decode.cu", "paged4_prefill.cu"]
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC", "-Xcompiler", "-fvisibility=hidden", "--expt-relaxed-constexpr"]


def _nvcc() -> str:
    cand = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "bin", "nvcc")
    return cand if os.path.exists(cand) else "nvcc"


def needs_build() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if not f.endswith(".cpp")] + [os.path.join(ROOT, "include", "moqae.h")]
    return any(os.path.getmtime(d) > t for d in deps)


def _torch_include() -> str:
    """The headers of the torch that is imported here, or an empty string where it has none, or none for CUDA."""
    try:
        import torch
    except ImportError:
        return ""
    path = os.path.join(os.path.dirname(torch.__file__), "include")
    needed = (("torch", "csrc", "autograd", "python_variable.h"), ("c10", "cuda", "CUDAStream.h"))
    return path if all(os.path.exists(os.path.join(path, *n)) for n in needed) else ""


def marshal_key() -> str:
    """What the argument marshalling module is built against: layouts of tensors and objects are compiled into it."""
    import torch
    return f"torch {torch.__version__}, C++ ABI {int(torch._C._GLIBCXX_USE_CXX11_ABI)}, {sys.implementation.cache_tag}"


def build_marshal(force: bool = False) -> str:
    """The argument marshalling module, against the torch that is imported here; again if it was built against another."""
    src = os.path.join(CSRC, "marshal.cpp")
    deps = [src, os.path.join(ROOT, "include", "moqae.h")]
    key = marshal_key()
    if not force and os.path.exists(MARSHAL) and all(os.path.getmtime(d) <= os.path.getmtime(MARSHAL) for d in deps):
        with open(MARSHAL, "rb") as f:
            if key.encode() in f.read():
                return MARSHAL
    import sysconfig

    import torch
    t, headers = os.path.dirname(torch.__file__), _torch_include()
    cuda = os.environ.get("CUDA_HOME", "/usr/local/cuda")
    include = [os.path.join(ROOT, "include"), headers, os.path.join(headers, "torch", "csrc", "api", "include"),
               sysconfig.get_paths()["include"], os.path.join(cuda, "include")]
    subprocess.check_call(["g++", f'-DMOQAE_BUILT_FOR="{key}"', "-O2", "-std=c++17", "-shared", "-fPIC", "-fvisibility=hidden",
                           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", *[f"-I{d}" for d in include], src, "-o", MARSHAL,
                           "-L" + os.path.join(t, "lib"), "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10", "-lc10_cuda"])
    return MARSHAL


def build(force: bool = False, verbose: bool = False) -> str:
    """The C library, which needs nvcc alone, then the Python module, where torch and its headers are there."""
    if force or needs_build():
        _build_library(verbose)
    if _torch_include():
        build_marshal(force)
    else:
        sys.stderr.write(f"torch or its headers are not here: {os.path.basename(MARSHAL)} is left out (the C library does not need it)\n")
    return LIB


def _build_library(verbose: bool) -> None:
    objs = []
    bdir = os.path.join(HERE, "_build")
    os.makedirs(bdir, exist_ok=True)
    procs = []
    for src in SOURCES:
        obj = os.path.join(bdir, src.replace(".cu", ".o"))
        cmd = [_nvcc(), *NVCC_FLAGS, "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-c",
               os.path.join(CSRC, src), "-o", obj]
        if verbose:
            cmd.insert(1, "-Xptxas")
            cmd.insert(2, "-v")
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
        objs.append(obj)
    for src, p in procs:
        out, _ = p.communicate()
        if verbose or p.returncode != 0:
            sys.stderr.write(out)
        if p.returncode != 0:
            raise RuntimeError(f"nvcc failed on {src}")
    cmd = [_nvcc(), "-shared", "-o", LIB, *objs, "-Xcompiler", "-fPIC", "-cudart", "static"]
    subprocess.check_call(cmd)


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
