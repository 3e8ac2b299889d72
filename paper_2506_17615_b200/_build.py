"""In-tree build of the CUDA library for sm_100a (nvcc cross-compiles without a GPU)."""
import fcntl
import os
import shutil
import subprocess
import sys
import sysconfig

_HERE = os.path.dirname(os.path.abspath(__file__))
_CSRC = os.path.join(_HERE, "csrc")
SOURCES = [os.path.join(_CSRC, name) for name in ("equarx_host.cu", "feedforward_host.cu", "norm_host.cu",
                                                    "adapter_host.cu")]
DEPENDS = SOURCES + [os.path.join(_CSRC, name) for name in ("equarx_kernels.cuh", "equarx_internal.h", "tensor_ops.cuh",
                                                            "feedforward_kernels.cuh", "elements.cuh", "host_common.h",
                                                            "norm_kernels.cuh", "adapter_kernels.cuh",
                                                            "adapter_tiles.cuh", "host_maps.h")] + \
    [os.path.join(os.path.dirname(_HERE), "include", "equarx.h")]
LIB = os.path.join(_HERE, "libequarx.so")
TORCH_SOURCE = os.path.join(_CSRC, "feedforward_torch.cpp")
TORCH_MODULE = os.path.join(_HERE, "_feedforward" + (sysconfig.get_config_var("EXT_SUFFIX") or ".so"))

NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC", "-shared", "--threads", "0"]


def find_nvcc():
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    return None


def is_stale():
    if not os.path.exists(LIB):
        return True
    built = os.path.getmtime(LIB)
    return any(os.path.getmtime(p) > built for p in DEPENDS)


def build(force=False, verbose=False):
    """Compile libequarx.so next to this file; returns its path.  EQUARX_LIBRARY=<path> in the
    environment selects an already built library instead (nothing is compiled then)."""
    prebuilt = os.environ.get("EQUARX_LIBRARY")
    if prebuilt and not force:
        if not os.path.exists(prebuilt):
            raise RuntimeError(f"EQUARX_LIBRARY={prebuilt} does not exist")
        return prebuilt
    if not force and not is_stale():
        return LIB
    nvcc = find_nvcc()
    if nvcc is None:
        raise RuntimeError("libequarx.so is missing or out of date and nvcc was not found; "
                           "the CUDA library cannot be built and there is no fallback")
    # several processes (one per GPU under torchrun) may import at once: one builds, the others wait
    with open(LIB + ".lock", "w") as lock:
        fcntl.flock(lock, fcntl.LOCK_EX)
        try:
            if force or is_stale():
                tmp = f"{LIB}.{os.getpid()}.tmp"
                cmd = [nvcc] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + ["-o", tmp] + SOURCES
                subprocess.run(cmd, check=True)
                os.replace(tmp, LIB)
        finally:
            fcntl.flock(lock, fcntl.LOCK_UN)
    return LIB


def find_cuda_home():
    for cand in (os.environ.get("CUDA_HOME"), os.path.dirname(os.path.dirname(find_nvcc() or "")), "/usr/local/cuda"):
        if cand and os.path.exists(os.path.join(cand, "include", "cuda_runtime_api.h")):
            return cand
    raise RuntimeError("the CUDA headers were not found; set CUDA_HOME")


def torch_stamp():
    """what a module compiled against torch's headers depends on, beside its sources"""
    import torch
    return f"{torch.__version__} {torch.version.git_version} cxx11={int(torch.compiled_with_cxx11_abi())} {sys.version}"


def torch_module_stale():
    """Missing, older than its sources, or compiled against another torch or Python than this one: by their
    versions, since an older torch installed over a newer one has older files."""
    sources = (TORCH_SOURCE, os.path.join(os.path.dirname(_HERE), "include", "equarx.h"))
    if not os.path.exists(TORCH_MODULE) or any(os.path.getmtime(p) > os.path.getmtime(TORCH_MODULE) for p in sources):
        return True
    try:
        with open(TORCH_MODULE + ".stamp") as f:
            return f.read() != torch_stamp()
    except OSError:
        return True


def build_torch_module(force=False):
    """Compile the extension module behind feedforward.py (torch tensors in and out); returns its path.  It
    depends on the library's header, not on the library, and on the installed torch."""
    import torch
    if force or torch_module_stale():
        with open(TORCH_MODULE + ".lock", "w") as lock:
            fcntl.flock(lock, fcntl.LOCK_EX)
            try:
                if force or torch_module_stale():
                    root = os.path.dirname(torch.__file__)
                    include, lib = os.path.join(root, "include"), os.path.join(root, "lib")
                    tmp, stamp = f"{TORCH_MODULE}.{os.getpid()}.tmp", f"{TORCH_MODULE}.stamp.{os.getpid()}.tmp"
                    subprocess.run([os.environ.get("CXX") or "g++", "-O2", "-std=c++17", "-shared", "-fPIC",
                                    f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}",
                                    "-I", sysconfig.get_paths()["include"], "-I", include,
                                    "-I", os.path.join(include, "torch", "csrc", "api", "include"),
                                    "-I", os.path.join(find_cuda_home(), "include"), "-o", tmp, TORCH_SOURCE,
                                    "-L", lib, "-ltorch_python", "-ltorch", "-ltorch_cpu", "-ltorch_cuda", "-lc10", "-lc10_cuda",
                                    # torch's own C++ runtime, by name: where only the static one can be
                                    # linked, a second copy in the process breaks its streams
                                    "-l:libstdc++.so.6", f"-Wl,-rpath,{lib}"], check=True)
                    with open(stamp, "w") as f:
                        f.write(torch_stamp())
                    os.replace(tmp, TORCH_MODULE)
                    os.replace(stamp, TORCH_MODULE + ".stamp")
            finally:
                fcntl.flock(lock, fcntl.LOCK_UN)
    return TORCH_MODULE
