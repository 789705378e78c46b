"""Build libpqadc.so (hand-written HIP for gfx950) in-tree with hipcc, and the binding's extension module with g++."""
import glob
import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libpqadc.so")
VIEWS = os.path.join(HERE, "tensor_views.so")

FLAGS = ["-O3", "--offload-arch=gfx950", "-std=c++17", "-fPIC", "-fno-gpu-rdc",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-Wall", "-Wno-unused-command-line-argument", "-I", os.path.join(ROOT, "include"), "-I", CSRC]


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.hip")))


def build_lib(verbose=False, extra=()):
    """Compile every .hip under csrc/ and link them into libpqadc.so.  Always recompiles."""
    objs = []
    procs = []
    for src in sources():
        obj = os.path.splitext(src)[0] + ".o"
        cmd = ["hipcc", *FLAGS, *extra, "-c", src, "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        procs.append((src, subprocess.Popen(cmd, stderr=subprocess.PIPE, text=True)))
        objs.append(obj)
    for src, p in procs:
        _, err = p.communicate()
        err = "\n".join(l for l in err.splitlines() if "packed-fp32-ops" not in l and l.strip())
        if p.returncode != 0:
            raise RuntimeError(f"hipcc failed on {src}:\n{err}")
        if err and verbose:
            print(err, file=sys.stderr)
    subprocess.run(["hipcc", "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB, *objs], check=True)
    return LIB


def build_views():
    """Compile csrc/tensor_views.cpp into an extension module.  Always recompiles."""
    import torch
    from torch.utils import cpp_extension
    # (its own headers before torch's; torch's libraries are in the process by the time the module is imported)
    includes = [os.path.join(ROOT, "include"), sysconfig.get_paths()["include"], *cpp_extension.include_paths()]
    libs = cpp_extension.library_paths()
    subprocess.run(["g++", "-O2", "-fPIC", "-std=c++17", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
                    *(f"-I{p}" for p in includes), os.path.join(CSRC, "tensor_views.cpp"), "-o", VIEWS,
                    *(f"-L{p}" for p in libs), "-ltorch_python", "-ltorch_cpu", "-lc10"], check=True)
    return VIEWS


if __name__ == "__main__":
    print(build_lib(verbose=True, extra=sys.argv[1:]))
    print(build_views())
