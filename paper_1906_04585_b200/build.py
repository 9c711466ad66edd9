"""Build libgala.so (sm_100a) in-tree with nvcc.

`python -m paper_1906_04585_b200.build` or `build()`; the shared object is
written next to this file so that it travels with the source tree.  Beside it
comes the compiled torch front end (csrc/front.cpp), which needs g++ and the
headers of an installed torch; where it cannot be built that is said, and
everything works without it.
"""
import glob
import importlib.metadata
import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libgala.so")
# The same sources with GALA_CROSS_CHECK defined: the only library in which the environment variable
# GALA_CONV_LEGACY selects the earlier convolution products (a second implementation that one test compares
# with the oracle).  Nothing but that test loads it.
CHECK_LIB = os.path.join(HERE, "libgala_check.so")
# The short way from torch tensors to the sequence-policy operators (csrc/front.cpp), a CPython module for one interpreter
# and one torch; FRONT_STAMP holds the version of the torch that it was compiled against.
FRONT_LIB = os.path.join(HERE, "_front" + (sysconfig.get_config_var("EXT_SUFFIX") or ".so"))
FRONT_STAMP = os.path.join(HERE, "_build", "front.torch")
FRONT_SRC = os.path.join(CSRC, "front.cpp")
NVCC = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")

FLAGS = [
    "-O3", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo",
    "-Xcompiler", "-fPIC",
    "-I", os.path.join(ROOT, "include"), "-I", CSRC,
]


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def _older(built, deps) -> bool:
    if not all(os.path.exists(p) for p in built):
        return True
    t = min(os.path.getmtime(p) for p in built)
    return any(os.path.getmtime(p) > t for p in deps)


def _stale() -> bool:
    headers = glob.glob(os.path.join(CSRC, "*.h")) + glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(os.path.join(ROOT, "include", "*.h"))
    return _older((LIB, CHECK_LIB), sources() + headers)


def _torch_version() -> str:
    try:
        return importlib.metadata.version("torch")
    except importlib.metadata.PackageNotFoundError:
        return ""


def _front_stale() -> bool:
    if _older((FRONT_LIB, FRONT_STAMP), [FRONT_SRC] + glob.glob(os.path.join(ROOT, "include", "*.h"))):
        return True
    with open(FRONT_STAMP) as f:
        return f.read() != _torch_version()


def _front_command(out: str):
    """g++ command of the torch front end: linked to the torch that this interpreter imports and to libgala.so beside it."""
    import torch
    from torch.utils import cpp_extension
    cuda = os.path.dirname(os.path.dirname(NVCC))
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-D_GLIBCXX_USE_CXX11_ABI=%d" % int(torch._C._GLIBCXX_USE_CXX11_ABI),
           '-DGALA_TORCH_VERSION="%s"' % torch.__version__, "-I" + os.path.join(ROOT, "include"), "-I" + sysconfig.get_paths()["include"], "-isystem", os.path.join(cuda, "include")]
    for d in cpp_extension.include_paths():
        cmd += ["-isystem", d]
    cmd += [FRONT_SRC, "-o", out, "-L" + HERE, "-l:libgala.so", "-Wl,-rpath,$ORIGIN"]
    for d in cpp_extension.library_paths():
        cmd += ["-L" + d, "-Wl,-rpath," + d]
    return cmd + ["-lc10", "-lc10_cuda", "-ltorch_cpu", "-ltorch", "-ltorch_python"]


def _build_front() -> None:
    """The torch front end; a failure is reported and leaves none, so that sequence.py goes its Python way."""
    tmp = FRONT_LIB + ".tmp.%d" % os.getpid()
    try:
        r = subprocess.run(_front_command(tmp), stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
        why = "" if r.returncode == 0 else r.stdout.strip()[-2000:] or "the compiler ended with %d" % r.returncode
    except (ImportError, OSError) as e:      # no torch, no g++, no headers
        why = "%s: %s" % (type(e).__name__, e)
    if not why:
        os.replace(tmp, FRONT_LIB)
        os.makedirs(os.path.dirname(FRONT_STAMP), exist_ok=True)
        with open(FRONT_STAMP, "w") as f:
            f.write(_torch_version())
        return
    for left in (tmp, FRONT_LIB):
        if os.path.exists(left):
            os.remove(left)
    sys.stderr.write("== %s is not built, calls on torch tensors go through Python: %s\n" % (os.path.basename(FRONT_LIB), why))


def build(force: bool = False, verbose: bool = False) -> str:
    if force or _stale():
        _build_library(verbose)
    if force or _front_stale():
        _build_front()
    return LIB


def _build_library(verbose: bool) -> None:
    objs = []
    procs = []
    os.makedirs(os.path.join(HERE, "_build"), exist_ok=True)
    for src in sources():
        obj = os.path.join(HERE, "_build", os.path.basename(src) + ".o")
        objs.append(obj)
        cmd = [NVCC] + FLAGS + (["-Xptxas", "-v"] if verbose else []) + ["-c", src, "-o", obj]
        procs.append((src, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    api_src = os.path.join(CSRC, "api.cu")
    api_check = os.path.join(HERE, "_build", "api.cu.check.o")
    procs.append((api_src + " (cross-check)", subprocess.Popen(
        [NVCC] + FLAGS + ["-DGALA_CROSS_CHECK", "-c", api_src, "-o", api_check],
        stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    failed = False
    for src, p in procs:
        out, _ = p.communicate()
        if p.returncode != 0 or verbose:
            sys.stderr.write("== %s\n%s\n" % (os.path.basename(src), out))
        failed |= p.returncode != 0
    if failed:
        raise RuntimeError("nvcc failed")
    tmp = LIB + ".tmp.%d" % os.getpid()
    subprocess.check_call([NVCC, "-shared", "-o", tmp] + objs + ["-gencode", "arch=compute_100a,code=sm_100a"])
    os.replace(tmp, LIB)
    check_objs = [api_check if os.path.basename(o) == "api.cu.o" else o for o in objs]
    tmp = CHECK_LIB + ".tmp.%d" % os.getpid()
    subprocess.check_call([NVCC, "-shared", "-o", tmp] + check_objs + ["-gencode", "arch=compute_100a,code=sm_100a"])
    os.replace(tmp, CHECK_LIB)


if __name__ == "__main__":
    print(build(force=True, verbose="-v" in sys.argv))
