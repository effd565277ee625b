"""Builds the CUDA library ``libbrisk.so`` in-tree for sm_103a with nvcc, and the binding's module ``_marshal``.

Each translation unit compiles in parallel, then one shared link. The runtime
is linked statically, so the library loads on a machine without a GPU driver
(the driver is opened on first use). ``_marshal`` is a module of the interpreter, compiled on its headers and
torch's, beside the library; it is compiled anew for another interpreter, which its name tells, and another torch.
"""
import os
import shutil
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libbrisk.so")
MARSHAL = os.path.join(HERE, "_marshal" + sysconfig.get_config_var("EXT_SUFFIX"))
MARSHAL_OF = os.path.join(BUILD, "marshal.torch")   # the version of the torch that it is for
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
FLAGS = ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC", "--expt-relaxed-constexpr",
         "-Xptxas", "-warn-spills"]


def nvcc() -> str:
    for cand in (os.environ.get("NVCC"), shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found")


def sources():
    return sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".cu"))


def current(target, deps):
    return os.path.exists(target) and all(os.path.getmtime(p) <= os.path.getmtime(target) for p in deps)


def run(cmd, what):
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"{what}:\n{r.stdout}\n{r.stderr}")
    return r.stdout + r.stderr


def is_for(version):
    if not os.path.exists(MARSHAL_OF):
        return False
    with open(MARSHAL_OF) as f:
        return f.read() == version


def build_marshal(src):
    import torch
    at = os.path.dirname(torch.__file__)
    cuda = os.path.join(os.path.dirname(nvcc()), "..", "include")
    tmp = MARSHAL + ".tmp"
    run([shutil.which(os.environ.get("CXX", "g++")) or "c++", "-O2", "-std=c++17", "-fPIC", "-shared", src, "-o", tmp,
         f"-I{sysconfig.get_paths()['include']}", f"-I{at}/include", f"-I{cuda}",
         f"-L{at}/lib", "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10", "-lc10_cuda"],
        f"compiling {src} failed")
    os.replace(tmp, MARSHAL)


def build(verbose: bool = False, force: bool = False) -> str:
    import torch
    header = os.path.join(HERE, "..", "include", "brisk.h")
    marshal = os.path.join(CSRC, "marshal.cpp")
    os.makedirs(BUILD, exist_ok=True)
    with ThreadPoolExecutor(max_workers=1) as ex:
        other = None
        if force or not is_for(torch.__version__) or not current(MARSHAL, [marshal, header, __file__]):
            other = ex.submit(build_marshal, marshal)
        path = build_library(header, verbose, force)
        if other:
            other.result()
            with open(MARSHAL_OF, "w") as f:
                f.write(torch.__version__)
    return path


def build_library(header, verbose, force):
    srcs = sources()
    deps = srcs + [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".cuh", ".h"))]
    if not force and current(LIB, [*deps, header, __file__]):
        return LIB
    cc = nvcc()

    def compile_one(src):
        obj = os.path.join(BUILD, os.path.basename(src)[:-3] + ".o")
        cmd = [cc, *ARCH, *FLAGS, "-c", src, "-o", obj]
        said = run(cmd, f"nvcc failed for {src}")
        if verbose and said:
            print(said, file=sys.stderr)
        return obj

    with ThreadPoolExecutor(max_workers=min(8, len(srcs))) as ex:
        objs = list(ex.map(compile_one, srcs))
    tmp = LIB + ".tmp"
    run([cc, *ARCH, "-shared", "-cudart", "static", "-o", tmp, *objs], "link failed")
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv, force="-f" in sys.argv))
