"""Build of libcoverprune.so: every CUDA source compiled for sm_103a (in
parallel, one nvcc per translation unit) and linked in-tree into
paper_2608_13226_gb300/_build/, with coverprune_torch beside it, the module that
takes tensors to the decoding model's calls.  No CMake, no setuptools.  Run as a
file with --library it builds the library alone, without Python's or torch's headers."""
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


def _newer(out, deps) -> bool:
    return os.path.exists(out) and all(os.path.getmtime(p) <= os.path.getmtime(out) for p in deps)


def library_up_to_date() -> bool:
    heads = [glob.glob(os.path.join(d, e)) for d, e in ((CSRC, "*.cuh"), (CSRC, "*.h"), (INCLUDE, "*.h"))]
    return _newer(LIB, _sources() + sum(heads, []) + [__file__])


def module_up_to_date() -> bool:
    deps = glob.glob(os.path.join(CSRC, "*.cpp")) + glob.glob(os.path.join(INCLUDE, "*.h")) + [__file__]
    return _newer(TORCH_LIB, deps) and _compiled_against() == _torch_id()


def up_to_date() -> bool:
    return library_up_to_date() and module_up_to_date()


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


def _start(cmd):
    return subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)


def _finish(procs, verbose):
    failed = []
    for src, p in procs:
        out, _ = p.communicate()
        if verbose and out:
            sys.stdout.write(out)
        if p.returncode != 0:
            failed.append((src, out))
    if failed:
        msg = "\n".join(f"--- {s}\n{o}" for s, o in failed)
        raise RuntimeError(f"compilation failed:\n{msg}")


def _link(out, cmd):
    """Links to a file of this process's own and moves it to its place."""
    tmp = out + f".tmp{os.getpid()}"
    r = subprocess.run([*cmd, "-o", tmp], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}")
    os.replace(tmp, out)


def _build_library(verbose, extra_flags):
    cc = nvcc()
    objs, procs = [], []
    for src in _sources():
        objs.append(os.path.join(BUILD, os.path.basename(src)[:-3] + ".o"))
        procs.append((src, _start([cc, *ARCH, *NVCC_FLAGS, *extra_flags, "-c", src, "-o", objs[-1]])))
    _finish(procs, verbose)
    _link(LIB, [cc, *ARCH, "-shared", *objs])


def build(force: bool = False, verbose: bool = False, extra_flags=(), module: bool = True) -> str:
    """Compile and link; returns the library path.  The library needs nvcc alone; module=False
    leaves out the module for PyTorch, which needs Python's and torch's headers."""
    os.makedirs(BUILD, exist_ok=True)
    library = force or not library_up_to_date()
    if not module:
        if library:
            _build_library(verbose, extra_flags)
        return LIB
    if not library and not force and module_up_to_date():
        return LIB
    # the module compiles beside the library; whatever fails of it, the library is there
    src, obj, failed = os.path.join(CSRC, "torch_binding.cpp"), os.path.join(BUILD, "torch_binding.o"), None
    cxx = shutil.which("g++") or "c++"
    try:
        comp, link = _torch_flags()
        proc = (src, _start([cxx, *comp, "-c", src, "-o", obj]))
    except Exception as e:
        failed = e
    if library:
        _build_library(verbose, extra_flags)
    if failed:
        raise RuntimeError(f"the module for PyTorch cannot be compiled: {failed}") from failed
    _finish([proc], verbose)
    _link(TORCH_LIB, [cxx, "-shared", obj, *link])
    with open(TORCH_MARK, "w") as f:
        f.write(_torch_id())
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv,
                extra_flags=["-Xptxas", "-v"] if "--ptxas" in sys.argv else [], module="--library" not in sys.argv))
