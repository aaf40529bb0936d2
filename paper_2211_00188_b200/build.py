"""Builds libadacgd.so (sm_100a) in-tree with nvcc, and with the host compiler the Python binding of the training operators,
_train_binding.so.  `python -m paper_2211_00188_b200.build`."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
import sysconfig
from importlib import metadata
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libadacgd.so")
BINDING = os.path.join(PKG, "_train_binding.so")
BINDING_SOURCE = "adacgd_train_binding.cpp"
STAMP = BINDING + ".for"   # the interpreter and torch the binding was compiled for
SOURCES = ["adacgd_api.cu", "adacgd_compress.cu", "adacgd_small.cu", "adacgd_noalloc.cu", "adacgd_gradient.cu",
           "adacgd_train.cu", "adacgd_train_norm.cu", "adacgd_train_loss.cu", "adacgd_train_embed.cu", "adacgd_train_rotary.cu",
           "adacgd_train_attention.cu", "adacgd_train_attention_mma.cu"]


def nvcc_path() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found")


def _older(target: str, sources) -> bool:
    return not os.path.exists(target) or any(os.path.getmtime(p) > os.path.getmtime(target) for p in sources)


def _headers():
    include = os.path.join(ROOT, "include")
    return [os.path.join(include, f) for f in os.listdir(include)]


def library_is_stale() -> bool:
    return _older(LIB, [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f != BINDING_SOURCE] + _headers())


def binding_target() -> str:
    """What the binding's object code depends on besides its source: it uses CPython's and torch's binary interfaces."""
    return f"{sysconfig.get_config_var('SOABI')}, torch {metadata.version('torch')}"


def binding_built_for():
    """The binding_target() that _train_binding.so was compiled for; None if that is not known."""
    try:
        with open(STAMP) as f:
            return f.read().strip()
    except OSError:
        return None


def binding_is_stale() -> bool:
    return _older(BINDING, [os.path.join(CSRC, BINDING_SOURCE)] + _headers()) or binding_built_for() != binding_target()


def needs_build() -> bool:
    return library_is_stale() or binding_is_stale()


def build(force: bool = False, verbose: bool = False) -> str:
    if force or library_is_stale():
        build_library(verbose)
    if force or binding_is_stale():
        build_binding()
    return LIB


def build_library(verbose: bool = False) -> str:
    flags = ["-O3", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo",
             "-fmad=false",  # every binary32 operation of the bit-exact path is a single rounding
             "-Xcompiler", "-fPIC", "-I", os.path.join(ROOT, "include"), "-I", CSRC]
    flags += os.environ.get("ADACGD_NVCC_FLAGS", "").split()  # extra compiler flags, e.g. -D switches
    if verbose:
        flags += ["-Xptxas", "-v"]
    objdir = os.path.join(PKG, "_build")
    os.makedirs(objdir, exist_ok=True)
    nvcc = nvcc_path()

    def compile_one(src):   # one translation unit -> one object, the units in parallel
        obj = os.path.join(objdir, src.replace(".cu", ".o"))
        res = subprocess.run([nvcc] + flags + ["-c", os.path.join(CSRC, src), "-o", obj], capture_output=True, text=True)
        return src, obj, res

    with ThreadPoolExecutor(max_workers=len(SOURCES)) as pool:
        done = list(pool.map(compile_one, SOURCES))
    for src, obj, res in done:
        if verbose or res.returncode != 0:
            sys.stderr.write(res.stdout + res.stderr)
        if res.returncode != 0:
            raise RuntimeError(f"nvcc failed on {src}")
    res = subprocess.run([nvcc, "-shared", "-gencode", "arch=compute_100a,code=sm_100a", "-o", LIB] + [o for _, o, _ in done],
                         capture_output=True, text=True)
    if res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
        raise RuntimeError("linking libadacgd.so failed")
    return LIB


def build_binding() -> str:
    """The extension module that checks torch tensors and calls libadacgd.so (which it finds beside itself)."""
    import torch

    root = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(os.path.realpath(nvcc_path())))
    include = [os.path.join(ROOT, "include"), sysconfig.get_paths()["include"], os.path.join(root, "include"),
               os.path.join(root, "include", "torch", "csrc", "api", "include"), os.path.join(cuda, "include")]
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}"]
    cmd += [f"-I{d}" for d in include] + [os.path.join(CSRC, BINDING_SOURCE), "-o", BINDING, "-L" + os.path.join(root, "lib"),
                                          "-ltorch_python", "-ltorch_cpu", "-ltorch", "-lc10", "-lc10_cuda", "-L" + PKG, "-l:libadacgd.so",
                                          "-Wl,-rpath,$ORIGIN"]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        sys.stderr.write(res.stdout + res.stderr)
        raise RuntimeError(f"{cmd[0]} failed on {BINDING_SOURCE}")
    with open(STAMP, "w") as f:
        f.write(binding_target() + "\n")
    return BINDING


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
