"""Build the HIP library ``libsvfsim.so`` for gfx950 with hipcc.

The library holds every kernel of the simulator and the host runtime behind
the C ABI of ``include/svfsim.h``, the paged cache's operators
(``include/svfkv.h``), the scores of answers (``include/svflogprob.h``) and the host-side exact optimum of tiny burst instances
(``include/svfopt.h``).  It is built in-tree so that the same file
is loaded by the tests, the smoke check and the benchmark.  ``_svfbinding.so`` beside it
is the binding to torch of the cache's calls and the scores; without a compiler or headers for it the library is built all the same.
"""

import os
import shutil
import subprocess
import sys
import warnings
from typing import Optional

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD = os.path.join(ROOT, "_build")
LIB = os.path.join(PKG, "libsvfsim.so")

ARCH = os.environ.get("SVFSIM_ARCH", "gfx950")
# Packed FP32 instructions are kept out of every code object.  Uniform
# branches are left as scalar branches rather than structured with lane masks
# (the simulation kernels are bound by scalar instruction issue).
GPU_FLAGS = ["-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
             "-mllvm", "-structurizecfg-skip-uniform-regions"]
# The cache's kernels are ordinary vector code: the same without the branch flag.
KV_GPU_FLAGS = GPU_FLAGS[:4]
KV_KERNELS = ("svf_kv_append", "svf_kv_rows", "svf_kv_chunk", "svf_kv_evict", "svf_logprob")
HOST = ("svf_kv", "svf_logprob_host", "svf_runtime", "svf_opt")
COMMON = ["-O3", "-std=c++17", "-fPIC", "-Wall", "-I", INCLUDE, "-I", CSRC]


def _run(cmd):
    subprocess.check_call(cmd)


def _run_all(cmds):
    """Runs them side by side, at most one for each CPU; all have ended when it raises."""
    running, failed, todo = [], None, list(cmds)
    while running or todo:
        while todo and failed is None and len(running) < max(1, min(os.cpu_count() or 1, 16)):
            running.append((todo[0], subprocess.Popen(todo.pop(0))))
        if not running:
            break
        cmd, p = running.pop(0)
        if p.wait() != 0 and failed is None:
            failed = subprocess.CalledProcessError(p.returncode, cmd)
    if failed is not None:
        raise failed


def build(verbose: bool = False) -> str:
    os.makedirs(BUILD, exist_ok=True)
    gpu = [(name, KV_GPU_FLAGS) for name in KV_KERNELS] + [(name, GPU_FLAGS) for name in ("svf_kernels", "svf_noalloc")]
    objects = [os.path.join(BUILD, name + ".o") for name in [n for n, _ in gpu] + list(HOST)]
    _run_all([["hipcc", f"--offload-arch={ARCH}", *COMMON, *flags, "-c", os.path.join(CSRC, name + ".hip"),
               "-o", os.path.join(BUILD, name + ".o")] for name, flags in gpu]
             + [["hipcc", *COMMON, "-c", os.path.join(CSRC, name + ".cpp"), "-o", os.path.join(BUILD, name + ".o")]
                for name in HOST])
    tmp = LIB + ".tmp"
    _run(["hipcc", f"--offload-arch={ARCH}", "-shared", "-fPIC", *objects, "-pthread", "-o", tmp])
    os.replace(tmp, LIB)
    build_binding()
    if verbose:
        print(LIB)
    return LIB


# What looks at torch's tensors for the cache's calls, against the headers and libraries of the torch that is installed.
BINDING = os.path.join(PKG, "_svfbinding.so")


def build_binding() -> Optional[str]:
    """None, with a warning and without the file of an earlier build, where the compiler or one of the headers is not there: the
    library serves without it, only slower calls from Python go through it."""
    import sysconfig

    try:
        import torch
    except ImportError:
        torch = None
    python, at = sysconfig.get_path("include"), os.path.dirname(torch.__file__) if torch else ""
    include = [os.path.join(at, "include"), os.path.join(at, "include", "torch", "csrc", "api", "include"), python]
    missing = [what for what, there in (("g++", shutil.which("g++")), ("Python.h", os.path.exists(os.path.join(python, "Python.h"))),
                                        ("torch", torch), ("torch's headers", torch and os.path.isdir(include[1]))) if not there]
    if missing:
        if os.path.exists(BINDING):
            os.remove(BINDING)
        warnings.warn(f"the binding to torch is not built: no {', no '.join(missing)}", RuntimeWarning, stacklevel=2)
        return None
    tmp = BINDING + ".tmp"
    _run(["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
          f'-DSVF_TORCH_VERSION="{torch.__version__}"',
          "-I", INCLUDE, *[x for i in include for x in ("-isystem", i)], os.path.join(CSRC, "svf_binding.cpp"), "-o", tmp,
          "-L", PKG, "-l:libsvfsim.so", "-L", os.path.join(at, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10",
          "-Wl,-rpath,$ORIGIN"])
    os.replace(tmp, BINDING)
    return BINDING


# The runtime's host code under the address and undefined-behaviour
# sanitizers (device code is not instrumented: each flag goes to the host
# compilation only), for the ABI test driver of tests/native.
SAN_HOST = ["-Xarch_host", "-fsanitize=address,undefined", "-Xarch_host", "-fno-sanitize-recover=all",
            "-Xarch_host", "-fno-omit-frame-pointer"]
SAN_EXE = os.path.join(BUILD, "abi_asan")


def build_abi_sanitized(verbose: bool = False) -> str:
    """Link tests/native/abi_asan_main.cpp and a sanitized build of the
    runtime with the kernel objects of ``build()`` into ``_build/abi_asan``."""
    kern_o = os.path.join(BUILD, "svf_kernels.o")
    na_o = os.path.join(BUILD, "svf_noalloc.o")
    if not (os.path.exists(kern_o) and os.path.exists(na_o)):
        build()
    flags = ["-O1", "-g", "-std=c++17", "-fPIC", "-Wall", "-I", INCLUDE, "-I", CSRC]
    rt_o = os.path.join(BUILD, "svf_runtime_san.o")
    drv_o = os.path.join(BUILD, "abi_asan_main.o")
    _run(["hipcc", *flags, *SAN_HOST, "-c", os.path.join(CSRC, "svf_runtime.cpp"), "-o", rt_o])
    _run(["hipcc", *flags, *SAN_HOST, "-c", os.path.join(ROOT, "tests", "native", "abi_asan_main.cpp"),
          "-o", drv_o])
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    tmp = SAN_EXE + ".tmp"
    _run([os.path.join(rocm, "llvm", "bin", "clang++"), "-fsanitize=address,undefined", drv_o, rt_o,
          kern_o, na_o, "-L", os.path.join(rocm, "lib"), "-lamdhip64",
          "-Wl,-rpath," + os.path.join(rocm, "lib"), "-pthread", "-o", tmp])
    os.replace(tmp, SAN_EXE)
    if verbose:
        print(SAN_EXE)
    return SAN_EXE


if __name__ == "__main__":
    build(verbose=True)
    sys.exit(0)
