"""Build libmok.so (the C-ABI CUDA library) in-tree with nvcc for sm_100a, and _binding.so (its C++ entry points for torch
tensors) with g++.

`python -m paper_2609_36070_b200.build [--force] [--verbose]`.  nvcc cross-compiles without a GPU.
"""
import glob
import importlib.metadata
import os
import subprocess
import sys
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libmok.so")
BINDING = os.path.join(PKG, "_binding.so")
BINDING_SRC = os.path.join(CSRC, "binding.cpp")
BINDING_FOR = os.path.join(PKG, "build", "binding.torch")       # the torch and Python that _binding.so was compiled against
NVCC = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")

FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
         "-Xcompiler", "-fPIC", "-I", os.path.join(ROOT, "include"), "-I", CSRC]


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def _stale():
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = sources() + glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(os.path.join(ROOT, "include", "*.h"))
    return any(os.path.getmtime(d) > t for d in deps)


def build_binding(force: bool = False) -> str:
    """The Python extension module, linked against libmok.so beside it and against torch's libraries (loaded by torch)."""
    deps = [BINDING_SRC, os.path.join(ROOT, "include", "mok.h")]
    wanted = f"torch {importlib.metadata.version('torch')}, Python {sys.version.split()[0]}"
    built = ""
    if os.path.exists(BINDING_FOR):
        with open(BINDING_FOR) as f:
            built = f.read()
    if (not force and built == wanted and os.path.exists(BINDING) and
            all(os.path.getmtime(d) <= os.path.getmtime(BINDING) for d in deps)):
        return BINDING
    import torch
    site = os.path.join(os.path.dirname(torch.__file__), "")
    cuda = os.path.dirname(os.path.dirname(NVCC))
    include = [os.path.join(ROOT, "include"), site + "include", site + "include/torch/csrc/api/include",
               os.path.join(cuda, "include"), sysconfig.get_paths()["include"]]
    libs = ["c10", "c10_cuda", "torch", "torch_cpu", "torch_cuda", "torch_python"]
    subprocess.run(["g++", "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
                    *(f"-I{d}" for d in include), BINDING_SRC, "-o", BINDING + ".tmp", f"-L{site}lib", *(f"-l{n}" for n in libs),
                    f"-L{PKG}", "-l:libmok.so", "-Wl,-rpath,$ORIGIN"], check=True)
    os.replace(BINDING + ".tmp", BINDING)
    os.makedirs(os.path.dirname(BINDING_FOR), exist_ok=True)
    with open(BINDING_FOR, "w") as f:
        f.write(wanted)
    return BINDING


def build(force: bool = False, verbose: bool = False) -> str:
    if force or _stale():
        build_library(verbose)
    build_binding(force)
    return LIB


def build_library(verbose: bool = False) -> str:
    objdir = os.path.join(PKG, "build")
    os.makedirs(objdir, exist_ok=True)
    objs = []
    procs = []
    for src in sources():
        obj = os.path.join(objdir, os.path.basename(src)[:-3] + ".o")
        cmd = [NVCC, *FLAGS, "-c", src, "-o", obj]
        if verbose:
            cmd.insert(1, "-Xptxas")
            cmd.insert(2, "-v")
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
        objs.append(obj)
    failed = False
    for src, p in procs:
        out, _ = p.communicate()
        if out.strip() and (verbose or p.returncode):
            print(f"--- {os.path.basename(src)}\n{out}", file=sys.stderr)
        failed |= p.returncode != 0
    if failed:
        raise RuntimeError("nvcc failed")
    subprocess.run([NVCC, "-shared", "-gencode", "arch=compute_100a,code=sm_100a", "-o", LIB + ".tmp", *objs],
                   check=True)
    os.replace(LIB + ".tmp", LIB)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="--verbose" in sys.argv))
