"""Compile the CUDA library for sm_103a (in-tree, no cmake).

Each translation unit is compiled in parallel with ``-fmad=false`` (every
float64 multiply and add rounds once, as the objective's bit-exactness needs)
and linked into ``_build/libe2ga.so`` with the static CUDA runtime, which takes nvcc and
gcc.  ``_build/e2binding.so`` is the Python module of the calls whose time is the host's
(csrc/binding.cpp), for the Python and the torch that are there; where it cannot be built
the library does without it, and so do the calls.
"""
from __future__ import annotations

import concurrent.futures as cf
import importlib.util
import os
import re
import shutil
import subprocess
import sys
import sysconfig
import warnings

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
OUT_DIR = os.path.join(HERE, "_build")
LIB = os.path.join(OUT_DIR, "libe2ga.so")
BINDING = os.path.join(OUT_DIR, "e2binding.so")
BUILT_FOR = os.path.join(OUT_DIR, "e2binding.txt")
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
FLAGS = ["-O3", "-std=c++17", "-lineinfo", "-fmad=false", "-Xcompiler", "-fPIC", "-I", INCLUDE,
         "-I", CSRC]


def _nvcc():
    for c in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if c and os.path.exists(c):
            return c
    raise RuntimeError("nvcc not found")


def sources():
    return sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".cu"))


def _older(target, deps):
    return not os.path.exists(target) or any(os.path.getmtime(d) > os.path.getmtime(target) for d in deps)


def _headers():
    return [os.path.join(INCLUDE, f) for f in ("e2ga.h", "e2ops.h")]


def _stale():
    return _older(LIB, sources() + [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".cuh")] + _headers())


def _torch():
    """Where torch is installed, None where it is not (it is not imported)."""
    spec = importlib.util.find_spec("torch")
    return spec.submodule_search_locations[0] if spec and spec.submodule_search_locations else None


def binding_for():
    """What the module is built for: this Python and the torch that is installed (None: none is)."""
    try:
        with open(os.path.join(_torch() or "", "version.py")) as f:
            version = re.search(r"__version__ = '(.*)'", f.read())
    except OSError:
        return None
    return version and f"{sys.implementation.cache_tag}, torch {version[1]}"


def binding_built_for():
    """What the module that is there was built for; None where there is none."""
    if not os.path.exists(BINDING) or not os.path.exists(BUILT_FOR):
        return None
    with open(BUILT_FOR) as f:
        return f.read()


def _binding_stale():
    want = binding_for()
    return want is not None and (binding_built_for() != want or _older(BINDING, _headers() + [os.path.join(CSRC, "binding.cpp")]))


def _compile_binding():
    """The module's object, against the torch that is installed; returns what the link takes."""
    torch = _torch()
    cuda = os.path.dirname(os.path.dirname(os.path.realpath(_nvcc())))
    obj = os.path.join(OUT_DIR, "binding.o")
    includes = [INCLUDE, os.path.join(torch, "include"), os.path.join(torch, "include", "torch", "csrc", "api", "include"),
                os.path.join(cuda, "include"), sysconfig.get_paths()["include"]]
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", *(f"-I{i}" for i in includes), "-c", os.path.join(CSRC, "binding.cpp"), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"g++ failed for binding.cpp:\n{r.stderr}")
    libs = [f"-L{os.path.join(torch, 'lib')}", "-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch_python"]
    return ["-shared", obj, f"-L{OUT_DIR}", "-l:libe2ga.so", *libs, "-Wl,-rpath,$ORIGIN"]


def build(force: bool = False, verbose: bool = False, extra=()) -> str:
    os.makedirs(OUT_DIR, exist_ok=True)
    with cf.ThreadPoolExecutor(max_workers=1) as ex:
        binding = ex.submit(_compile_binding) if _binding_stale() or force and binding_for() else None
        if force or _stale():
            _build_library(verbose, extra)
        if binding:
            _link_binding(binding)
    return LIB


def _link_binding(compiled):
    """The module, from what its compilation gives; a warning where that failed."""
    tmp = BINDING + ".tmp"
    if os.path.exists(BUILT_FOR):
        os.remove(BUILT_FOR)               # (an older module is not taken for this one)
    try:
        r = subprocess.run(["g++", "-o", tmp, *compiled.result()], capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"link failed:\n{r.stderr}")
    except (OSError, RuntimeError) as e:
        warnings.warn(f"e2binding.so was not built, calls take some 15 us longer: {e}")
        return
    os.replace(tmp, BINDING)
    with open(BUILT_FOR + ".tmp", "w") as f:
        f.write(binding_for())
    os.replace(BUILT_FOR + ".tmp", BUILT_FOR)


def _build_library(verbose, extra):
    srcs = sources()
    objs = [os.path.join(OUT_DIR, os.path.basename(s)[:-3] + ".o") for s in srcs]
    nvcc = _nvcc()

    def compile_one(pair):
        src, obj = pair
        cmd = [nvcc, *ARCH, *FLAGS, *extra, "-c", src, "-o", obj]
        if verbose:
            cmd.insert(1, "-Xptxas=-v")
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"nvcc failed for {src}:\n{r.stderr}")
        return r.stderr

    with cf.ThreadPoolExecutor(max_workers=len(srcs)) as ex:
        logs = list(ex.map(compile_one, zip(srcs, objs)))
    if verbose:
        for l in logs:
            print(l)
    tmp = LIB + ".tmp"
    r = subprocess.run([nvcc, *ARCH, "-shared", "-o", tmp, *objs], capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stderr}")
    os.replace(tmp, LIB)


if __name__ == "__main__":
    import sys
    print(build(force=True, verbose="-v" in sys.argv))
