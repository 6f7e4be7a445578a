"""Builds the HIP library in-tree for gfx950, and the compiled part of its Python binding (a few seconds each)."""
import glob
import os
import subprocess
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libnestedfp.so")
MARSHAL = os.path.join(PKG, "_marshal.so")          # csrc/marshal.cpp, imported by binding.py

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # keep the compiler from emitting packed-FP32 VALU forms
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wno-unused-command-line-argument",
]


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.hip")))


def lib_path():
    return LIB


def is_stale():
    if not (os.path.exists(LIB) and os.path.exists(MARSHAL)):
        return True
    t = min(os.path.getmtime(LIB), os.path.getmtime(MARSHAL))
    deps = sources() + glob.glob(os.path.join(CSRC, "*.cpp")) + glob.glob(os.path.join(CSRC, "*.h")) + glob.glob(os.path.join(CSRC, "*.inc")) + glob.glob(os.path.join(ROOT, "include", "*.h"))
    return any(os.path.getmtime(d) > t for d in deps)


def _run(cmd, verbose):
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    out = "\n".join(l for l in res.stdout.splitlines() if "packed-fp32-ops" not in l)
    if res.returncode != 0:
        raise RuntimeError("%s failed:\n%s" % (os.path.basename(cmd[0]), out))
    if verbose and out.strip():
        print(out, flush=True)


def _marshal_command():
    import torch

    home = os.path.dirname(torch.__file__)
    return [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared",
            "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch.compiled_with_cxx11_abi(),
            "-I", sysconfig.get_paths()["include"], "-I", os.path.join(home, "include"),
            "-I", os.path.join(home, "include", "torch", "csrc", "api", "include"),
            os.path.join(CSRC, "marshal.cpp"), "-o", MARSHAL,
            "-L", os.path.join(home, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10"]


def build_library(verbose=False, binding=True):
    """Compiles every source to an object of its own (in parallel, under _build/) and links them; beside it, unless `binding` is
    false, the compiled part of the Python binding.  That one needs Python's and torch's headers and a host compiler, which the library
    does not: where it fails the library is built all the same, and the error comes afterwards."""
    from concurrent.futures import ThreadPoolExecutor

    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    objdir = os.path.join(PKG, "_build")
    os.makedirs(objdir, exist_ok=True)
    srcs = sources()
    objs = [os.path.join(objdir, os.path.basename(s)[:-4] + ".o") for s in srcs]
    cmds = [[hipcc] + HIPCC_FLAGS + ["-I", os.path.join(ROOT, "include"), "-c", s, "-o", o]
            for s, o in zip(srcs, objs)]
    jobs = min(len(cmds) + bool(binding), int(os.environ.get("MAX_JOBS", "0")) or os.cpu_count() or 1)
    with ThreadPoolExecutor(max_workers=jobs) as pool:
        marshal = pool.submit(lambda: _run(_marshal_command(), verbose)) if binding else None
        list(pool.map(lambda c: _run(c, verbose), cmds))
    _run([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB] + objs, verbose)
    if marshal is not None and marshal.exception() is not None:
        raise RuntimeError("the library is built (%s), the compiled part of the Python binding is not" % LIB) from marshal.exception()
    return LIB


if __name__ == "__main__":
    import sys

    build_library(verbose=True, binding="--no-binding" not in sys.argv[1:])
    print("built", LIB)
