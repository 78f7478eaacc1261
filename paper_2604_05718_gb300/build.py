"""Builds libmpm.so (the C-ABI library) in-tree for sm_103a with nvcc.

Each .cu file under csrc/ is compiled in parallel to an object file in
_build/, then linked into paper_2604_05718_gb300/libmpm.so with the CUDA
runtime linked statically and only the mpm_* symbols exported.  Beside it,
csrc/blocks_binding.cpp becomes the extension module _blocks, the Python
binding of the encoder-block entry points.  That takes torch's C++ headers and a
host compiler; where it fails, the library is there all the same, and the
block operators raise at their first call.
"""

from __future__ import annotations

import concurrent.futures
import glob
import os
import shutil
import subprocess
import sysconfig
import warnings

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
BUILD = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libmpm.so")
# The same sources with the device timeline compiled in (-DMPM_TRACE); see
# mpm_trace_read in include/mpm.h.  Used by `bench.py --timeline` only.
BUILD_TRACE = os.path.join(PKG, "_build_trace")
LIB_TRACE = os.path.join(PKG, "libmpm_trace.so")
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
NVCC_FLAGS = ARCH + ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC,-fvisibility=hidden",
                     "-I", os.path.join(ROOT, "include"), "-I", CSRC]


BINDING_SRC = os.path.join(CSRC, "blocks_binding.cpp")
BINDING = os.path.join(PKG, "_blocks" + sysconfig.get_config_var("EXT_SUFFIX"))


def nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found: the MPM library needs the CUDA toolkit to build")


def _headers() -> list:
    return glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(os.path.join(CSRC, "*.h")) + \
        [os.path.join(ROOT, "include", "mpm.h")]


def _stale(target: str, deps: list) -> bool:
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(d) > t for d in deps)


def _run(cmd: list) -> None:
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"command failed ({res.returncode}): {' '.join(cmd)}\n{res.stdout}\n{res.stderr}")


def _binding_command(out: str) -> list:
    """g++ over the binding, against the torch that runs this."""
    import torch

    root = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(os.path.realpath(nvcc())))
    include = [os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include"),
               os.path.join(cuda, "include"), sysconfig.get_paths()["include"], os.path.join(ROOT, "include")]
    lib = os.path.join(root, "lib")
    return [os.environ.get("CXX", "g++"), "-shared", "-fPIC", "-O2", "-std=c++17", "-fvisibility=hidden",
            f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}", BINDING_SRC, "-o", out] + \
        [f"-I{d}" for d in include] + [f"-L{lib}", "-ltorch_python", "-ltorch_cuda", "-ltorch_cpu", "-ltorch", "-lc10",
                                       "-lc10_cuda", f"-Wl,-rpath,{lib}"]


def _binding_key() -> str:
    """What the binding is built for, next to its sources: this torch, whose ABI it has, and the command."""
    import torch

    return " ".join([torch.__version__, str(torch.version.git_version)] + _binding_command(""))


def _binding_stale() -> bool:
    if _stale(BINDING, [BINDING_SRC, os.path.join(ROOT, "include", "mpm.h")]):
        return True
    try:
        with open(os.path.join(BUILD, "blocks_binding.txt")) as f:
            return f.read() != _binding_key()
    except Exception:  # never noted, or no torch here
        return True


def _build_binding() -> None:
    tmp = BINDING + ".tmp"
    try:
        _run(_binding_command(tmp))
        with open(os.path.join(BUILD, "blocks_binding.txt"), "w") as f:
            f.write(_binding_key())
    except Exception as e:  # no torch, no compiler, or one that fails: the merge needs none of them
        if os.path.exists(BINDING):
            os.remove(BINDING)
        warnings.warn(f"the binding of the block operators was not built: {e}", RuntimeWarning)
    else:
        os.replace(tmp, BINDING)


def build(force: bool = False, extra_flags: list | None = None, trace: bool = False) -> str:
    """Compiles and links libmpm.so (libmpm_trace.so with trace=True) and the
    binding module if any source changed; returns the library's path."""
    build_dir, lib_path = (BUILD_TRACE, LIB_TRACE) if trace else (BUILD, LIB)
    os.makedirs(build_dir, exist_ok=True)
    srcs = sorted(glob.glob(os.path.join(CSRC, "*.cu")))
    headers = _headers()
    flags = NVCC_FLAGS + (["-DMPM_TRACE"] if trace else []) + list(extra_flags or [])
    jobs = []
    objs = []
    for src in srcs:
        obj = os.path.join(build_dir, os.path.basename(src)[:-3] + ".o")
        objs.append(obj)
        if force or _stale(obj, [src] + headers):
            jobs.append([nvcc(), "-c", src, "-o", obj] + flags)
    compiled = bool(jobs)
    bind = not trace and (force or _binding_stale())
    with concurrent.futures.ThreadPoolExecutor(max_workers=8) as ex:
        binding = ex.submit(_build_binding) if bind else None
        list(ex.map(_run, jobs))
    if binding is not None:
        binding.result()
    if force or compiled or _stale(lib_path, objs):
        tmp = lib_path + ".tmp"
        _run([nvcc(), "-shared", "-o", tmp] + objs + ARCH +
             ["-cudart", "static", "-Xlinker", "--version-script=" + os.path.join(CSRC, "exports.map")])
        os.replace(tmp, lib_path)
    return lib_path


if __name__ == "__main__":
    print(build(force=True))
