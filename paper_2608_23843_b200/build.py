"""Builds libpkv.so (the C-ABI CUDA library) in-tree with nvcc for sm_100a, and _pkvcall, a module of the interpreter that builds it through
which the Python binding makes the calls of a decode step (a C source against the library, gcc and Python's headers)."""
import glob
import os
import subprocess
import sys
import sysconfig
import tempfile
import warnings
from concurrent.futures import ThreadPoolExecutor

_HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(_HERE)
CSRC = os.path.join(_HERE, "csrc")
LIB = os.path.join(_HERE, "libpkv.so")
# (the name has the interpreter's ABI in it: another one neither takes it for its own nor finds it fresh)
CALL, CALL_SOURCE = os.path.join(_HERE, "_pkvcall" + (sysconfig.get_config_var("EXT_SUFFIX") or ".so")), os.path.join(CSRC, "pkv_call.c")
NVCC = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def build_call(force=False):
    """Compile the binding's calls; returns the module's path.  Where that fails (no C compiler, no Python headers) it warns and returns None: the library is
    complete without, and the binding makes its calls through ctypes."""
    deps = [CALL_SOURCE, os.path.join(ROOT, "include", "pkv.h")]
    if not force and os.path.exists(CALL) and all(os.path.getmtime(f) <= os.path.getmtime(CALL) for f in deps):
        return CALL
    tmp = CALL + ".tmp.%d" % os.getpid()
    old = os.path.join(_HERE, "_pkvcall.so")             # (a name that any interpreter would import)
    if old != CALL and os.path.exists(old):
        os.remove(old)
    try:
        subprocess.run([os.environ.get("CC", "gcc"), "-O2", "-std=c11", "-Wall", "-shared", "-fPIC", "-I", sysconfig.get_path("include"), "-I", os.path.join(ROOT, "include"),
                        CALL_SOURCE, "-o", tmp, "-L", _HERE, "-l:libpkv.so", "-Wl,-rpath,$ORIGIN"], check=True)
    except (OSError, subprocess.CalledProcessError) as e:
        if os.path.exists(CALL):                         # (of another source: not to be called)
            os.remove(CALL)
        warnings.warn("%s was not built (%s): calls of a decode step go through ctypes, 3 us more each" % (os.path.basename(CALL), e))
        return None
    os.replace(tmp, CALL)
    return CALL


def _stale():
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = sources() + glob.glob(os.path.join(CSRC, "*.h")) + glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(os.path.join(ROOT, "include", "*.h"))
    return any(os.path.getmtime(f) > t for f in deps)


def build(force=False, verbose=False):
    """Compile every .cu under csrc/ into one shared library, and the binding's calls; returns the library's path."""
    if not force and not _stale():
        build_call()
        return LIB
    # one nvcc per source, side by side: the kernels' many shapes take minutes one after the other
    flags = ["-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC",
             "-I", os.path.join(ROOT, "include"), "-I", CSRC]
    if verbose:
        flags += ["-Xptxas", "-v"]
    tmp = LIB + ".tmp.%d" % os.getpid()
    with tempfile.TemporaryDirectory() as folder:
        objects = [os.path.join(folder, os.path.basename(src) + ".o") for src in sources()]

        def compile_one(pair):
            subprocess.run([NVCC, *flags, "-c", pair[0], "-o", pair[1]], check=True)

        with ThreadPoolExecutor(max(1, os.cpu_count() or 1)) as pool:
            list(pool.map(compile_one, zip(sources(), objects)))
        subprocess.run([NVCC, *flags, "-shared", *objects, "-o", tmp], check=True)
    os.replace(tmp, LIB)
    build_call(force=True)
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose="-v" in sys.argv))
