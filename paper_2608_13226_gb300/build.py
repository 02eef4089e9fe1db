"""Build of libcoverprune.so: every CUDA source compiled for sm_103a (in
parallel, one nvcc per translation unit) and linked in-tree into
paper_2608_13226_gb300/_build/, with coverprune_torch beside it, the module that
takes tensors to the decoding model's calls.  No CMake, no setuptools."""
from __future__ import annotations

import glob
import os
import shutil
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(BUILD, "libcoverprune.so")
TORCH_LIB = os.path.join(BUILD, "coverprune_torch.so")
TORCH_MARK = os.path.join(BUILD, "coverprune_torch.txt")  # what TORCH_LIB was compiled against
INCLUDE = os.path.join(os.path.dirname(HERE), "include")

ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
NVCC_FLAGS = ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC", "-Xcompiler", "-O2",
              "--expt-relaxed-constexpr", "-I" + INCLUDE]


def nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found: the CoverPrune CUDA library cannot be built")


def _sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def _deps():
    return _sources() + glob.glob(os.path.join(CSRC, "*.cuh")) + \
        glob.glob(os.path.join(CSRC, "*.h")) + glob.glob(os.path.join(CSRC, "*.cpp")) + glob.glob(os.path.join(INCLUDE, "*.h")) + [__file__]


def up_to_date() -> bool:
    if not os.path.exists(LIB) or not os.path.exists(TORCH_LIB):
        return False
    t = min(os.path.getmtime(LIB), os.path.getmtime(TORCH_LIB))
    return all(os.path.getmtime(p) <= t for p in _deps()) and _compiled_against() == _torch_id()


def _torch_id() -> str:
    """The interpreter and torch whose headers and layout a module depends on."""
    import torch
    return f"{torch.__version__} {os.path.dirname(torch.__file__)} {sys.implementation.cache_tag}"


def _compiled_against():
    try:
        with open(TORCH_MARK) as f:
            return f.read()
    except OSError:
        return None


def _torch_flags():
    """Compiler and linker flags of the module that takes tensors."""
    import torch
    at = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(os.path.realpath(nvcc())))
    inc = [os.path.join(at, "include"), os.path.join(at, "include", "torch", "csrc", "api", "include"),
           sysconfig.get_paths()["include"], os.path.join(cuda, "include"), INCLUDE]
    abi = int(torch._C._GLIBCXX_USE_CXX11_ABI)
    comp = ["-O2", "-std=c++17", "-fPIC", "-fvisibility=hidden", f"-D_GLIBCXX_USE_CXX11_ABI={abi}",
            *(f"-I{i}" for i in inc)]
    # torch's own libraries are loaded by the import of torch that comes first
    link = ["-L" + BUILD, "-l:" + os.path.basename(LIB), "-Wl,-rpath,$ORIGIN", "-L" + os.path.join(at, "lib"),
            "-ltorch_python", "-ltorch_cuda", "-ltorch_cpu", "-lc10_cuda", "-lc10"]
    return comp, link


def build(force: bool = False, verbose: bool = False, extra_flags=()) -> str:
    """Compile and link; returns the library path."""
    if not force and up_to_date():
        return LIB
    os.makedirs(BUILD, exist_ok=True)
    cc = nvcc()
    procs = []
    objs = []
    for src in _sources():
        obj = os.path.join(BUILD, os.path.basename(src)[:-3] + ".o")
        objs.append(obj)
        cmd = [cc, *ARCH, *NVCC_FLAGS, *extra_flags, "-c", src, "-o", obj]
        procs.append((src, cmd, subprocess.Popen(cmd, stdout=subprocess.PIPE,
                                                 stderr=subprocess.STDOUT, text=True)))
    comp, torch_link = _torch_flags()
    cxx = shutil.which("g++") or "c++"
    src = os.path.join(CSRC, "torch_binding.cpp")
    torch_obj = os.path.join(BUILD, "torch_binding.o")
    cmd = [cxx, *comp, "-c", src, "-o", torch_obj]
    procs.append((src, cmd, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT,
                                             text=True)))
    failed = []
    for src, cmd, p in procs:
        out, _ = p.communicate()
        if verbose and out:
            sys.stdout.write(out)
        if p.returncode != 0:
            failed.append((src, out))
    if failed:
        msg = "\n".join(f"--- {s}\n{o}" for s, o in failed)
        raise RuntimeError(f"compilation failed:\n{msg}")
    for out, link in ((LIB, [cc, *ARCH, "-shared", "-o", None, *objs]),
                      (TORCH_LIB, [cxx, "-shared", "-o", None, torch_obj, *torch_link])):
        tmp = out + f".tmp{os.getpid()}"
        link[link.index(None)] = tmp
        r = subprocess.run(link, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"link failed:\n{r.stdout}")
        os.replace(tmp, out)
    with open(TORCH_MARK, "w") as f:
        f.write(_torch_id())
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv,
                extra_flags=["-Xptxas", "-v"] if "--ptxas" in sys.argv else []))
