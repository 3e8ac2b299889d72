"""In-tree build of the CUDA library for sm_100a (nvcc cross-compiles without a GPU)."""
import fcntl
import os
import shutil
import subprocess
import sysconfig

_HERE = os.path.dirname(os.path.abspath(__file__))
_CSRC = os.path.join(_HERE, "csrc")
SOURCES = [os.path.join(_CSRC, "equarx_host.cu"), os.path.join(_CSRC, "feedforward_host.cu")]
DEPENDS = SOURCES + [os.path.join(_CSRC, name) for name in ("equarx_kernels.cuh", "equarx_internal.h", "tensor_ops.cuh",
                                                            "feedforward_kernels.cuh")] + \
    [os.path.join(os.path.dirname(_HERE), "include", "equarx.h")]
LIB = os.path.join(_HERE, "libequarx.so")
FASTCALL_SOURCE = os.path.join(_CSRC, "fastcall.c")
FASTCALL = os.path.join(_HERE, "_fastcall" + (sysconfig.get_config_var("EXT_SUFFIX") or ".so"))

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


def build_fastcall(force=False):
    """Compile the extension module that calls the feed-forward entry points without ctypes; returns its path.
    It depends on the header alone, not on the library, and needs a C compiler and Python's headers."""
    sources = (FASTCALL_SOURCE, os.path.join(os.path.dirname(_HERE), "include", "equarx.h"))

    def stale():
        return not os.path.exists(FASTCALL) or any(os.path.getmtime(p) > os.path.getmtime(FASTCALL) for p in sources)

    if force or stale():
        with open(FASTCALL + ".lock", "w") as lock:
            fcntl.flock(lock, fcntl.LOCK_EX)
            try:
                if force or stale():
                    tmp = f"{FASTCALL}.{os.getpid()}.tmp"
                    subprocess.run([os.environ.get("CC") or "gcc", "-O2", "-std=c11", "-Wall", "-shared", "-fPIC",
                                    "-I", sysconfig.get_paths()["include"], "-o", tmp, FASTCALL_SOURCE], check=True)
                    os.replace(tmp, FASTCALL)
            finally:
                fcntl.flock(lock, fcntl.LOCK_UN)
    return FASTCALL
