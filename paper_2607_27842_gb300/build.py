"""Builds libfeatfix.so (the C-ABI library) in-tree for sm_103a with nvcc.

Each translation unit under csrc/ is compiled to an object in parallel, then
the objects are linked into ``paper_2607_27842_gb300/libfeatfix.so``.  The
CUDA runtime is linked statically; the driver entry point used for TMA
descriptors is resolved at run time, so the library loads on a machine
without a GPU.  Beside it g++ builds ``_ops8.so``, the Python module that
marshals the 8-bit operators' arguments (csrc/py_ops8.cpp); it needs the headers of
PyTorch and Python, and where they are missing the library is built alone (a note
says so, and the 8-bit operators' Python calls raise).
"""

import concurrent.futures
import importlib.util
import os
import shutil
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
BUILD_DIR = os.path.join(ROOT, "_build")
LIB = os.path.join(HERE, "libfeatfix.so")

ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
FLAGS = ["-O3", "-std=c++17", "-lineinfo", "-Xcompiler", "-fPIC", "-Xcompiler", "-fvisibility=hidden",
         "--expt-relaxed-constexpr", "-I", os.path.join(ROOT, "include"), "-I", CSRC]
SOURCES = ["ff_elementwise.cu", "ff_simt.cu", "ff_gemm_tc.cu", "ff_attention.cu", "ff_attention_tc.cu", "ff_runtime.cu", "ff_ops.cu", "ff_noalloc.cu",
           "ff_rows8.cu", "ff_rope.cu", "ff_gemm8.cu", "ff_kv8.cu", "ff_kv_attention.cu", "ff_block_norms.cu"]


# the Python module that marshals the 8-bit operators' arguments (C++ only)
BINDING = "py_ops8.cpp"
BINDING_LIB = os.path.join(HERE, "_ops8.so")


def nvcc():
    path = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(path):
        raise RuntimeError("nvcc not found")
    return path


def _compile(src, extra):
    obj = os.path.join(BUILD_DIR, os.path.splitext(src)[0] + ".o")
    cmd = [nvcc()] + ARCH + FLAGS + extra + ["-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("nvcc failed on %s:\n%s\n%s" % (src, r.stdout, r.stderr))
    return obj, r.stderr


def _torch_dir():
    """PyTorch's folder (headers and libraries), found without importing it; None
    where it is not installed."""
    spec = importlib.util.find_spec("torch")
    return spec.submodule_search_locations[0] if spec and spec.submodule_search_locations else None


def _binding_lacks():
    """What the binding cannot be built without and is not there, or None."""
    if shutil.which("g++") is None:
        return "g++"
    t = _torch_dir()
    if t is None or not os.path.exists(os.path.join(t, "include", "torch", "csrc", "autograd", "python_variable.h")):
        return "PyTorch with its headers"
    if not os.path.exists(os.path.join(sysconfig.get_paths()["include"], "Python.h")):
        return "Python.h"
    return None


def _run(what, cmd):
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("%s failed:\n%s\n%s" % (what, r.stdout, r.stderr))


def _compile_binding():
    t = os.path.join(_torch_dir(), "include")
    cuda = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(nvcc()))), "include")
    obj = os.path.join(BUILD_DIR, "py_ops8.o")
    inc = [t, os.path.join(t, "torch", "csrc", "api", "include"), sysconfig.get_paths()["include"], cuda,
           os.path.join(ROOT, "include")]
    _run("g++ on " + BINDING, ["g++", "-O2", "-std=c++17", "-fPIC", "-fvisibility=hidden"] +
         [x for p in inc for x in ("-isystem" if p.startswith(t) else "-I", p)] +
         ["-c", os.path.join(CSRC, BINDING), "-o", obj])
    return obj


def _link_binding(obj):
    tmp = BINDING_LIB + ".tmp"
    _run("link of " + BINDING, ["g++", "-shared", "-o", tmp, obj, LIB, "-Wl,-rpath,$ORIGIN", "-L" +
                                os.path.join(_torch_dir(), "lib"), "-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_python"])
    os.replace(tmp, BINDING_LIB)


def build(verbose=False, extra=()):
    """Compile and link; returns the library path."""
    os.makedirs(BUILD_DIR, exist_ok=True)
    extra = list(extra)
    lacks = _binding_lacks()
    with concurrent.futures.ThreadPoolExecutor(max_workers=len(SOURCES) + 1) as ex:
        binding = None if lacks else ex.submit(_compile_binding)
        results = list(ex.map(lambda s: _compile(s, extra), SOURCES))
    objs = [o for o, _ in results]
    if verbose:
        for _, err in results:
            if err.strip():
                sys.stderr.write(err)
    tmp = LIB + ".tmp"
    cmd = [nvcc()] + ARCH + ["-shared", "-Xcompiler", "-fPIC", "-Xlinker", "-soname=libfeatfix.so", "-o", tmp] + objs + \
        ["-cudart", "static"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed:\n%s\n%s" % (r.stdout, r.stderr))
    os.replace(tmp, LIB)
    if lacks:
        if os.path.exists(BINDING_LIB):   # of another build: linked to what the library was then
            os.remove(BINDING_LIB)
        sys.stderr.write("%s is not built (%s is missing): no Python calls of the 8-bit operators\n" %
                         (os.path.basename(BINDING_LIB), lacks))
    else:
        _link_binding(binding.result())
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv, extra=["-Xptxas", "-v"] if "--ptxas" in sys.argv else []))
