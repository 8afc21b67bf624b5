"""Build libstr.so (the C-ABI CUDA library) in-tree with nvcc for sm_100a.

``python -m paper_2603_00198_b200.build`` compiles every ``csrc/*.cu`` into ``_build/*.o`` (in
parallel) and links ``paper_2603_00198_b200/libstr.so``, then compiles ``csrc/marshal.cpp`` (host code: the binding's argument
marshalling of the decode calls) into ``paper_2603_00198_b200/_marshal.so``.  No GPU is needed to build.
"""
import concurrent.futures
import glob
import os
import shutil
import subprocess
import sys
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
OBJ = os.path.join(ROOT, "_build")
LIB = os.path.join(PKG, "libstr.so")
MARSHAL = os.path.join(PKG, "_marshal.so")
BUILT_FOR = os.path.join(OBJ, "marshal.torch")

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-lineinfo", "-std=c++17",
    "-Xcompiler", "-fPIC", "-I" + os.path.join(ROOT, "include"), "-I" + CSRC,
]


def _deps_mtime():
    hdrs = glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(os.path.join(ROOT, "include", "*.h"))
    return max(os.path.getmtime(h) for h in hdrs)


def _compile(src, verbose):
    obj = os.path.join(OBJ, os.path.basename(src)[:-3] + ".o")
    if os.path.exists(obj) and os.path.getmtime(obj) >= max(os.path.getmtime(src), _deps_mtime()):
        return obj, ""
    cmd = ["nvcc"] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + ["-c", src, "-o", obj]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("nvcc failed for %s:\n%s" % (src, res.stderr))
    return obj, res.stderr


def _built_for():
    try:
        with open(BUILT_FOR) as f:
            return f.read()
    except OSError:
        return None


def _build_marshal(force):
    """The extension module links against torch's C++ libraries, which the process has loaded when it imports the module.  It is built
    anew for another torch, whose version is kept in the module (`built_for`, which the binding compares) and beside the objects."""
    import torch
    src = os.path.join(CSRC, "marshal.cpp")
    if not force and os.path.exists(MARSHAL) and os.path.getmtime(MARSHAL) >= max(os.path.getmtime(src), _deps_mtime()) and _built_for() == torch.__version__:
        return
    tdir = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(shutil.which("nvcc")))
    incs = [os.path.join(tdir, "include"), os.path.join(tdir, "include", "torch", "csrc", "api", "include"),
            sysconfig.get_paths()["include"], os.path.join(cuda, "include")]
    cmd = ["g++", "-O2", "-std=c++17", "-Wall", "-fPIC", "-shared", "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch.compiled_with_cxx11_abi(),
           '-DSTR_BUILT_FOR="%s"' % torch.__version__, "-I" + os.path.join(ROOT, "include")] + [a for i in incs for a in ("-isystem", i)]
    cmd += [src, "-o", MARSHAL, "-L" + os.path.join(tdir, "lib"), "-ltorch_python", "-ltorch_cpu", "-ltorch", "-lc10", "-lc10_cuda"]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("g++ failed for %s:\n%s" % (src, res.stderr))
    with open(BUILT_FOR, "w") as f:
        f.write(torch.__version__)


def build(force=False, verbose=False):
    os.makedirs(OBJ, exist_ok=True)
    srcs = sorted(glob.glob(os.path.join(CSRC, "*.cu")))
    if force:
        for o in glob.glob(os.path.join(OBJ, "*.o")):
            os.remove(o)
    with concurrent.futures.ThreadPoolExecutor(max_workers=os.cpu_count() or 4) as ex:
        results = list(ex.map(lambda s: _compile(s, verbose), srcs))
    objs = [o for o, _ in results]
    if verbose:
        for _, log in results:
            sys.stderr.write(log)
    if (not os.path.exists(LIB)) or any(os.path.getmtime(o) > os.path.getmtime(LIB) for o in objs):
        cmd = ["nvcc", "-shared", "-gencode", "arch=compute_100a,code=sm_100a", "-o", LIB] + objs
        subprocess.run(cmd, check=True)
    _build_marshal(force)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
