"""Builds libsubnetact.so (HIP kernels + C ABI) for gfx950 with hipcc, and the serving binding, in tree."""
import concurrent.futures as cf
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libsubnetact.so")
SERVING = os.path.join(HERE, "_serving.so")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = ["-O3", "--offload-arch=gfx950", "-fPIC", "-std=c++17", "-Wall", "-Wno-unused-function",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         # leading scalar kernel arguments arrive in registers
         "-mllvm", "-amdgpu-kernarg-preload-count=14"]


def sources():
    return sorted(f for f in os.listdir(CSRC) if f.endswith(".hip"))


def _compile(src):
    obj = os.path.join(OBJ, src[:-4] + ".o")
    cmd = [HIPCC, *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    err = "\n".join(l for l in r.stderr.splitlines() if "packed-fp32-ops" not in l)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed on {src}:\n{err}")
    if err.strip():
        sys.stderr.write(err + "\n")
    return obj


def build_library(verbose: bool = True) -> str:
    os.makedirs(OBJ, exist_ok=True)
    with cf.ThreadPoolExecutor(max_workers=6) as ex:
        objs = list(ex.map(_compile, sources()))
    r = subprocess.run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB, *objs],
                       capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed:\n" + r.stderr)
    if verbose:
        print(f"built {LIB}")
    return LIB


def build_serving(verbose: bool = True) -> str:
    """The serving operators' Python binding (host code only) against the built library and the installed torch.  The C ABI
    and the rest of the package do without it."""
    import sysconfig

    from torch.utils.cpp_extension import include_paths, library_paths
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    inc = [*include_paths(), os.path.join(rocm, "include"), sysconfig.get_paths()["include"]]
    lib = [d for p in (*library_paths(), os.path.join(rocm, "lib")) for d in ("-L" + p, "-Wl,-rpath," + p)]
    r = subprocess.run(["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", "-fvisibility=hidden", "-D__HIP_PLATFORM_AMD__", "-DUSE_ROCM",
                        *[x for p in inc for x in ("-isystem", p)], os.path.join(CSRC, "serving_py.cpp"), "-o", SERVING,
                        "-L" + HERE, "-l:libsubnetact.so", "-Wl,-rpath,$ORIGIN", *lib, "-lc10", "-lc10_hip", "-ltorch", "-ltorch_cpu", "-ltorch_python", "-lamdhip64"],
                       capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("serving binding failed:\n" + r.stderr)
    if r.stderr.strip():
        sys.stderr.write(r.stderr)
    if verbose:
        print(f"built {SERVING}")
    return SERVING


if __name__ == "__main__":
    build_library()
    try:
        import torch  # noqa: F401
    except ImportError as e:
        print(f"not built: {SERVING}, the serving operators' Python side, needs torch ({e})")
    else:
        build_serving()
