"""Build libpard.so in-tree with nvcc for sm_103a (GB300), and the module
that calls its tree operators on torch tensors.

Translation units are compiled in parallel and linked into
``paper_2504_18583_gb300/libpard.so``; ``csrc/torch_binding.cpp`` becomes
``_tree_ops*.so`` beside it, compiled by the host compiler against the installed
torch; without torch only the library is built, which needs none.  A rebuild
happens when a source or header is newer than they are, or torch is another one.
"""
from __future__ import annotations

import concurrent.futures as cf
import fcntl
import glob
import importlib.metadata
import importlib.util
import os
import shutil
import subprocess
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
BUILD = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libpard.so")
BINDING_SRC = os.path.join(CSRC, "torch_binding.cpp")
BINDING = os.path.join(PKG, "_tree_ops" + sysconfig.get_config_var("EXT_SUFFIX"))
BINDING_TORCH = os.path.join(BUILD, "torch_binding.torch")  # which torch it was compiled against

ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
NVCC_FLAGS = ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC", "--expt-relaxed-constexpr",
              "-I" + os.path.join(ROOT, "include")]


def nvcc() -> str:
    for cand in (os.environ.get("CUDA_HOME", ""), "/usr/local/cuda"):
        p = os.path.join(cand, "bin", "nvcc") if cand else ""
        if p and os.path.exists(p):
            return p
    p = shutil.which("nvcc")
    if not p:
        raise RuntimeError("nvcc not found: the CUDA toolkit is required to build libpard")
    return p


def _sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def _deps():
    return _sources() + glob.glob(os.path.join(CSRC, "*.h")) + glob.glob(os.path.join(CSRC, "*.cuh")) + \
        glob.glob(os.path.join(ROOT, "include", "*.h")) + [BINDING_SRC, os.path.abspath(__file__)]


def installed_torch():
    """Version and place of the torch that this Python would import, or None; torch is not imported for it."""
    spec = importlib.util.find_spec("torch")
    if spec is None:
        return None
    try:
        version = importlib.metadata.version("torch")
    except importlib.metadata.PackageNotFoundError:
        version = "unknown"
    return f"{version} {spec.origin}"


def up_to_date() -> bool:
    made = [LIB]
    torch = installed_torch()
    if torch is not None:
        made.append(BINDING)
        if not os.path.exists(BINDING_TORCH) or open(BINDING_TORCH).read() != torch:
            return False
    if not all(os.path.exists(p) for p in made):
        return False
    t = min(os.path.getmtime(p) for p in made)
    return all(os.path.getmtime(p) <= t for p in _deps())


def build(verbose: bool = False, extra_flags=()) -> str:
    """Compile every .cu under csrc/ and link libpard.so; returns its path.
    Processes that build at once (one per rank under torch.distributed.run)
    take a file lock, so one compiles and the others find it up to date."""
    if up_to_date() and not extra_flags:
        return LIB
    os.makedirs(BUILD, exist_ok=True)
    with open(os.path.join(BUILD, ".lock"), "w") as lock:
        fcntl.flock(lock, fcntl.LOCK_EX)
        try:
            if up_to_date() and not extra_flags:
                return LIB
            return _compile_and_link(verbose, extra_flags)
        finally:
            fcntl.flock(lock, fcntl.LOCK_UN)


def _compile_and_link(verbose: bool, extra_flags) -> str:
    cc = nvcc()

    def compile_one(src):
        obj = os.path.join(BUILD, os.path.basename(src) + ".o")
        cmd = [cc, *ARCH, *NVCC_FLAGS, *extra_flags, "-c", src, "-o", obj]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"nvcc failed on {os.path.basename(src)}:\n{r.stdout}\n{r.stderr}")
        if verbose and (r.stdout or r.stderr):
            print(r.stdout, r.stderr)
        return obj

    torch = installed_torch()
    with cf.ThreadPoolExecutor(max_workers=min(12, os.cpu_count() or 4)) as ex:
        binding = ex.submit(_compile_binding) if torch is not None else None
        objs = list(ex.map(compile_one, _sources()))
    tmp = LIB + ".tmp"
    r = subprocess.run([cc, *ARCH, "-shared", "-o", tmp, *objs, "-lcuda"], capture_output=True, text=True)
    if r.returncode != 0:
        # libcuda is only needed for symbol resolution at load; fall back to the stub
        stub = "/usr/local/cuda/lib64/stubs"
        r = subprocess.run([cc, *ARCH, "-shared", "-o", tmp, *objs, "-L" + stub, "-lcuda"],
                           capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, LIB)
    if binding is not None:  # (the library is there whatever becomes of it)
        _link_binding(binding.result())
        with open(BINDING_TORCH, "w") as f:
            f.write(torch)
    return LIB


def _run(cmd, what):
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"{what} failed:\n{r.stdout}\n{r.stderr}")


def _torch_dir():
    import torch
    return os.path.dirname(os.path.abspath(torch.__file__)), int(torch._C._GLIBCXX_USE_CXX11_ABI)


def _compile_binding() -> str:
    tdir, abi = _torch_dir()
    obj = os.path.join(BUILD, "torch_binding.o")
    cuda = os.path.dirname(os.path.dirname(nvcc()))
    _run(["g++", "-O2", "-std=c++20", "-fPIC", "-w", f"-D_GLIBCXX_USE_CXX11_ABI={abi}",
          "-I" + os.path.join(ROOT, "include"), "-I" + os.path.join(tdir, "include"),
          "-I" + os.path.join(tdir, "include", "torch", "csrc", "api", "include"),
          "-I" + os.path.join(cuda, "include"), "-I" + sysconfig.get_paths()["include"],
          "-c", BINDING_SRC, "-o", obj], "g++ on torch_binding.cpp")
    return obj


def _link_binding(obj: str) -> None:
    tdir, _ = _torch_dir()
    tmp = BINDING + ".tmp"
    _run(["g++", "-shared", "-o", tmp, obj, "-L" + PKG, "-l:libpard.so", "-L" + os.path.join(tdir, "lib"), "-lc10",
          "-lc10_cuda", "-ltorch_cpu", "-ltorch_python", "-Wl,-rpath,$ORIGIN", "-Wl,--allow-shlib-undefined"],
         "link of the torch binding")
    os.replace(tmp, BINDING)


if __name__ == "__main__":
    print(build(verbose=True))
