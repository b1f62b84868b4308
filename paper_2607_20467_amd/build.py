"""Build libdcl.so (HIP, gfx950) in-tree with hipcc. Runs on a machine without a GPU."""
import os
import shutil
import subprocess
import sys
import tempfile
import warnings
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libdcl.so")
SOURCES = ["abi.hip", "abi_serving.hip", "k_small.hip", "k_gemm.hip", "k_attn.hip", "k_pages.hip",
           "k_pages4.hip", "k_turn.hip", "k_heads.hip", "k_prompt.hip", "k_sample.hip"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
# (source, extra flags) of each object; the GEMM family's instantiations are spread over three of them
OBJECTS = [("k_gemm.hip", ["-DDCL_GEMM_PART=1"]), ("k_gemm.hip", ["-DDCL_GEMM_PART=2"]),
           ("k_gemm.hip", ["-DDCL_GEMM_PART=3"]), ("k_attn.hip", []), ("k_pages.hip", []), ("k_pages4.hip", []),
           ("k_turn.hip", []), ("k_heads.hip", []), ("k_prompt.hip", []),
           ("k_sample.hip", []), ("k_small.hip", []),
           ("abi.hip", []), ("abi_serving.hip", [])]
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # packed-FP32 instructions are kept out of generated code (all arithmetic here is scalar fp32)
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function", "-Wno-unused-variable",
]


def sources():
    return [os.path.join(CSRC, s) for s in SOURCES] + [os.path.join(CSRC, "operands.cpp")]


def operands_path() -> str:
    """The Python extension (csrc/operands.cpp: calls from Python in one step). It reads torch's objects as the headers lay them out,
    so that one for another torch or interpreter has another name and is never loaded."""
    import sysconfig

    import torch
    return os.path.join(HERE, "_operands." + str(torch.__version__) + sysconfig.get_config_var("EXT_SUFFIX"))


def drop_operands() -> None:
    """Extensions of any torch: each enters the library as the header was when it was built."""
    for name in os.listdir(HERE):
        if name.startswith("_operands.") and name.endswith(".so"):
            os.remove(os.path.join(HERE, name))


def build_operands(verbose: bool = False) -> str:
    """Compile the Python extension, host code against torch's headers. Returns its path."""
    import sysconfig

    import torch
    drop_operands()
    at, path = os.path.dirname(torch.__file__), operands_path()
    tmp = path + ".tmp%d" % os.getpid()
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall",
           "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch._C._GLIBCXX_USE_CXX11_ABI, "-D__HIP_PLATFORM_AMD__",
           "-isystem", os.path.join(at, "include"), "-isystem", sysconfig.get_paths()["include"],
           "-isystem", os.path.join(os.path.dirname(os.path.dirname(HIPCC)), "include"), "-I", os.path.join(ROOT, "include"),
           os.path.join(CSRC, "operands.cpp"), "-L", os.path.join(at, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10", "-o", tmp]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.check_call(cmd)
    os.replace(tmp, path)
    return path


def build(verbose: bool = False) -> str:
    """Compile every HIP source into libdcl.so, and the Python extension beside it (always recompiles). Returns the library path. What the
    extension lacks (a host compiler, torch's headers) costs the library nothing."""
    tmp = LIB + ".tmp%d" % os.getpid()
    objdir = tempfile.mkdtemp(prefix="dcl_build_")
    try:
        def compile_one(i):
            src, extra = OBJECTS[i]
            obj = os.path.join(objdir, "%d.o" % i)
            cmd = [HIPCC, *FLAGS, *extra, "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-c",
                   os.path.join(CSRC, src), "-o", obj]
            if verbose:
                print(" ".join(cmd), flush=True)
            subprocess.check_call(cmd)
            return obj
        with ThreadPoolExecutor(max_workers=min(len(OBJECTS) + 1, os.cpu_count() or 1)) as pool:
            extension = pool.submit(build_operands, verbose)
            objs = list(pool.map(compile_one, range(len(OBJECTS))))
        subprocess.check_call([HIPCC, "--offload-arch=gfx950", "-shared", *objs, "-o", tmp])
    except BaseException:
        drop_operands()                                 # the library stays as it was
        raise
    finally:
        shutil.rmtree(objdir, ignore_errors=True)
    os.replace(tmp, LIB)
    try:
        extension.result()
    except (OSError, subprocess.CalledProcessError, ImportError) as e:
        warnings.warn(f"the extension for calls from Python is not built: {e}", RuntimeWarning, stacklevel=2)
    return LIB


def is_stale() -> bool:
    if not os.path.exists(LIB) or not os.path.exists(operands_path()):
        return True
    t = min(os.path.getmtime(LIB), os.path.getmtime(operands_path()))
    deps = sources() + [os.path.join(CSRC, "dcl_internal.h"), os.path.join(CSRC, "gemm_tuned.inc"), os.path.join(CSRC, "pages_index.h"),
                        os.path.join(ROOT, "include", "dcl.h")]
    return any(os.path.getmtime(p) > t for p in deps)


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
