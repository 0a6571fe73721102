"""Build liblordba.so (sm_100a only) in-tree with nvcc, and the Python module _block next to it.

``python -m paper_2605_24058_b200.build``, or ``build_library()`` and ``build_binding()``.  Objects go
to ``paper_2605_24058_b200/_build``; the shared objects sit next to this file so
that they travel with a snapshot of the tree.  The library needs nvcc alone; the module also needs
the headers of torch and of Python.
"""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
BUILD = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "liblordba.so")
TESTHOOKS_LIB = os.path.join(PKG, "liblordba_testhooks.so")
SOURCES = ("api.cu", "block_api.cu", "elementwise.cu", "product.cu", "product_tile.cu", "product_stream.cu", "pack.cu", "fit.cu", "forward_fma.cu", "forward_tc.cu", "forward_mma.cu")
BINDING = os.path.join(PKG, "_block.so")       # Python module of csrc/binding.cpp
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC", "-Wno-deprecated-gpu-targets",
              "-I", os.path.join(ROOT, "include"), "-I", CSRC]


def _nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found; liblordba.so cannot be built")


def _newest_header() -> float:
    paths = [os.path.join(ROOT, "include", "lordba.h")]
    paths += [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".h", ".cuh"))]
    return max(os.path.getmtime(p) for p in paths)


def binding_made_for() -> str:
    """What the module is compiled against: an interpreter and a torch."""
    import torch
    return "Python %d.%d, torch %s" % (sys.version_info[0], sys.version_info[1], torch.__version__)


def _made_for_file() -> str:
    return os.path.join(BUILD, "_block.made_for")


def _binding_is_current() -> bool:
    newest = max(os.path.getmtime(os.path.join(CSRC, "binding.cpp")), os.path.getmtime(os.path.join(ROOT, "include", "lordba.h")))
    if not os.path.exists(BINDING) or os.path.getmtime(BINDING) < newest or not os.path.exists(_made_for_file()):
        return False
    with open(_made_for_file()) as f:
        return f.read() == binding_made_for()


def build_binding(force: bool = False) -> str:
    """Build the Python module ``_block`` (csrc/binding.cpp; g++ against the headers of the installed torch) where it is missing,
    older than its sources or made for another torch or Python."""
    if not force and _binding_is_current():
        return BINDING
    import sysconfig
    import torch
    home = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(_nvcc()))
    includes = [os.path.join(home, "include"), os.path.join(home, "include", "torch", "csrc", "api", "include"),
                sysconfig.get_paths()["include"], os.path.join(cuda, "include"), os.path.join(ROOT, "include")]
    os.makedirs(BUILD, exist_ok=True)
    tmp = BINDING + ".tmp.%d" % os.getpid()
    made_for = binding_made_for()
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", '-DMADE_FOR="%s"' % made_for,
           "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch._C._GLIBCXX_USE_CXX11_ABI]
    for d in includes:
        cmd += ["-isystem" if d.startswith(home) else "-I", d]
    cmd += [os.path.join(CSRC, "binding.cpp"), "-o", tmp, "-L", os.path.join(home, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda", "-ldl"]
    p = subprocess.run(cmd, capture_output=True, text=True)
    if p.returncode != 0:
        sys.stderr.write(p.stdout + p.stderr)
        raise RuntimeError("g++ failed: " + " ".join(cmd))
    os.replace(tmp, BINDING)
    with open(_made_for_file() + ".tmp.%d" % os.getpid(), "w") as f:
        f.write(made_for)
    os.replace(f.name, _made_for_file())
    return BINDING


def build_library(force: bool = False, verbose: bool = False, test_hooks: bool = False) -> str:
    """Build the library, and the Python module too where that can be had (a message says so where not: the
    library does without it, and the calls that need it raise).  test_hooks=True builds a second library, liblordba_testhooks.so, from
    the same sources with -DLORDBA_TEST_HOOKS (bounded device-side waits give up after about a
    millisecond, and lordba_test_skip_item makes one copy request go missing): only the test of
    the timeout path loads it; the product library never has the hooks."""
    build_dir = BUILD + ("_testhooks" if test_hooks else "")
    lib_path = TESTHOOKS_LIB if test_hooks else LIB
    extra = ["-DLORDBA_TEST_HOOKS"] if test_hooks else []
    os.makedirs(build_dir, exist_ok=True)
    nvcc = _nvcc()
    hdr = _newest_header()
    jobs = []
    for src in SOURCES:
        s = os.path.join(CSRC, src)
        o = os.path.join(build_dir, src + ".o")
        if force or not os.path.exists(o) or os.path.getmtime(o) < max(os.path.getmtime(s), hdr):
            cmd = [nvcc] + NVCC_FLAGS + extra + (["-Xptxas", "-v"] if verbose else []) + ["-c", s, "-o", o]
            jobs.append(cmd)

    def run(cmd):
        p = subprocess.run(cmd, capture_output=True, text=True)
        if verbose or p.returncode != 0:
            sys.stderr.write(p.stdout + p.stderr)
        if p.returncode != 0:
            raise RuntimeError("nvcc failed: " + " ".join(cmd))

    with ThreadPoolExecutor(max_workers=4) as ex:
        list(ex.map(run, jobs))
    objs = [os.path.join(build_dir, s + ".o") for s in SOURCES]
    if jobs or not os.path.exists(lib_path):
        tmp = lib_path + ".tmp.%d" % os.getpid()
        run([nvcc, "-shared", "-o", tmp] + objs + ["-Xlinker", "--exclude-libs=ALL"])
        os.replace(tmp, lib_path)
    if not test_hooks:
        try:
            build_binding(force)
        except Exception as e:          # no headers of torch or Python here
            sys.stderr.write("the Python module _block was not (re)built: %s\n" % e)
    return lib_path


if __name__ == "__main__":
    if "--test-hooks" not in sys.argv:
        build_binding(force="--force" in sys.argv)
    print(build_library(force="--force" in sys.argv, verbose="-v" in sys.argv,
                        test_hooks="--test-hooks" in sys.argv))
