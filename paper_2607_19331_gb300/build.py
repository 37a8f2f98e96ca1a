"""Build the CUDA library ``libiso_gb300.so`` in-tree for sm_103a, and the host
module ``_iso_train`` that marshals torch tensors for the training-step calls.

Each translation unit is compiled in parallel, then linked into a shared
library next to this file under ``_build/``.  Nothing is installed.  The library
takes nvcc alone; the host module takes g++ and torch, and is left out where
there is no torch (the C ABI needs neither).
"""
from __future__ import annotations

import concurrent.futures as cf
import os
import shutil
import subprocess
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(BUILD, "libiso_gb300.so")
BINDING = os.path.join(BUILD, "_iso_train.so")
STAMP = os.path.join(BUILD, "_iso_train.txt")    # the torch that BINDING was built for, and its commands
SOURCES = ["iso_api.cu", "iso_select.cu", "iso_apply.cu", "iso_merge.cu", "iso_block.cu", "iso_fused.cu",
           "iso_gemm.cu", "iso_frame.cu", "iso_range.cu", "iso_act.cu", "iso_wgrad.cu", "iso_embed.cu"]
HEADERS = ["iso_internal.cuh", "iso_kernels.cuh", "iso_gemm.cuh", "iso_train.cuh"]
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
FLAGS = ["-O3", "-lineinfo", "-std=c++17", "-static-global-template-stub=false", "-Xcompiler", "-fPIC,-ffp-contract=off",
         "--expt-relaxed-constexpr", "-I", os.path.join(ROOT, "include"), "-I", CSRC]


def nvcc() -> str:
    exe = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(exe):
        raise RuntimeError("nvcc not found: the CUDA toolkit is required to build libiso_gb300")
    return exe


def binding_commands(obj: str):
    """(compile, link) commands of the host module."""
    import torch
    root = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(os.path.realpath(nvcc())))
    cxx = shutil.which("g++") or "g++"
    inc = [os.path.join(ROOT, "include"), os.path.join(root, "include"),
           os.path.join(root, "include", "torch", "csrc", "api", "include"), os.path.join(cuda, "include"),
           "/usr/local/cuda/include", sysconfig.get_paths()["include"]]
    compile_ = [cxx, "-O2", "-std=c++17", "-fPIC", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
                *[x for i in inc if os.path.isdir(i) for x in ("-I", i)], "-c", os.path.join(CSRC, "train_binding.cpp"),
                "-o", obj]
    lib = os.path.join(root, "lib")
    link = [cxx, "-shared", obj, "-L", lib, "-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_python", "-L", BUILD,
            "-l:libiso_gb300.so", "-Wl,-rpath,$ORIGIN", f"-Wl,-rpath,{lib}"]
    return compile_, link


def _stale(target: str, deps) -> bool:
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(d) > t for d in deps)


def stamped_torch():
    """The torch version that the host module was built for, or None."""
    if not (os.path.exists(BINDING) and os.path.exists(STAMP)):
        return None
    with open(STAMP) as f:
        return f.readline().strip()


def _run(cmd) -> str:
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"compilation failed: {' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    return r.stderr


def _link(cmd, target: str) -> None:
    tmp = target + f".tmp{os.getpid()}"
    subprocess.check_call([*cmd, "-o", tmp])
    os.replace(tmp, target)


def build(force: bool = False, verbose: bool = False, extra=None) -> str:
    os.makedirs(BUILD, exist_ok=True)
    hdrs = [os.path.join(CSRC, h) for h in HEADERS] + [os.path.join(ROOT, "include", "iso.h")]
    objs, jobs = [], []
    for src in SOURCES:
        s = os.path.join(CSRC, src)
        o = os.path.join(BUILD, src.replace(".cu", ".o"))
        objs.append(o)
        if force or _stale(o, [s] + hdrs):
            cmd = [nvcc(), *ARCH, *FLAGS, *(extra or []), "-c", s, "-o", o]
            jobs.append(cmd)

    # the host module, again too where the torch or the commands are not those it was built with
    bobj = os.path.join(BUILD, "train_binding.o")
    try:
        import torch
        bcompile, blink = binding_commands(bobj)
        stamp = "\n".join([torch.__version__, " ".join(bcompile), " ".join(blink)]) + "\n"
    except ImportError:
        stamp = None
    if stamp is not None:
        bnew = force or _stale(bobj, [os.path.join(CSRC, "train_binding.cpp"), os.path.join(ROOT, "include", "iso.h")])
        if not bnew:
            bnew = not os.path.exists(STAMP) or open(STAMP).read() != stamp

    with cf.ThreadPoolExecutor(max_workers=len(SOURCES) + 1) as ex:
        binding = ex.submit(_run, bcompile) if stamp is not None and bnew else None
        errs = list(ex.map(_run, jobs))
        if force or jobs or _stale(LIB, objs):
            _link([nvcc(), *ARCH, "-shared", *objs, "-lcudart"], LIB)
        if binding is not None:       # its failure comes after the library, which does not need it
            errs.append(binding.result())
    if verbose:
        for err in errs:
            if err:
                print(err)
    if stamp is not None and (bnew or _stale(BINDING, [bobj])):
        _link(blink, BINDING)
        with open(STAMP, "w") as f:
            f.write(stamp)
    return LIB


if __name__ == "__main__":
    import sys
    print(build(force="--force" in sys.argv, verbose=True))
