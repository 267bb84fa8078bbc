"""Build libwavezip.so (HIP kernels + C ABI) for gfx950 with hipcc, and _serve.so, the Python binding of its serving
operators.

    python -m paper_2607_23265_amd.csrc.build      # or: python paper_2607_23265_amd/csrc/build.py

Compiles every .hip file of this directory to an object (in parallel) and
links them into paper_2607_23265_amd/libwavezip.so; serve_py.cpp, against
torch's headers, becomes paper_2607_23265_amd/_serve.so.  Always rebuilds.
"""
import concurrent.futures
import os
import shutil
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
PKG = os.path.dirname(HERE)
ROOT = os.path.dirname(PKG)
INCLUDE = os.path.join(ROOT, "include")
OBJDIR = os.path.join(ROOT, "_build", "wavezip")
LIB = os.path.join(PKG, "libwavezip.so")
BINDING = os.path.join(PKG, "_serve.so")
ARCH = "gfx950"

# -packed-fp32-ops: no v_pk_{add,mul,fma}_f32 in the generated code.
DEVICE_FLAGS = ["-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]
COMMON = ["-O3", "-std=c++17", "-fPIC", f"--offload-arch={ARCH}", "-I", INCLUDE, "-I", HERE,
          "-Wall", "-Wno-unused-function", "-Wno-unused-variable"]


def hipcc():
    path = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(path):
        raise RuntimeError("hipcc not found: the ROCm toolchain is required to build libwavezip.so")
    return path


def sources():
    return sorted(os.path.join(HERE, f) for f in os.listdir(HERE) if f.endswith(".hip"))


def _compile(src):
    obj = os.path.join(OBJDIR, os.path.basename(src)[:-4] + ".o")
    cmd = [hipcc(), *COMMON, *DEVICE_FLAGS, "-c", src, "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    # hipcc's host pass warns that it does not know the packed-fp32 feature: harmless
    msgs = "\n".join(l for l in (r.stdout + r.stderr).splitlines() if "packed-fp32-ops" not in l)
    if r.returncode != 0:
        raise RuntimeError(f"compiling {src} failed:\n{msgs}")
    return obj, msgs


def _compile_binding():
    """serve_py.cpp, host code alone, by the host compiler."""
    import torch
    src, obj = os.path.join(HERE, "serve_py.cpp"), os.path.join(OBJDIR, "serve_py.o")
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        raise RuntimeError("no C++ compiler (g++) for _serve.so")
    # (the HIP headers that torch's stream header includes want to be told their platform)
    rocm = os.path.dirname(os.path.dirname(os.path.realpath(hipcc())))
    system = [os.path.join(os.path.dirname(torch.__file__), "include"), os.path.join(rocm, "include"),
              sysconfig.get_paths()["include"]]
    cmd = [cxx, "-O2", "-std=c++17", "-fPIC", "-Wall", "-fvisibility=hidden", "-D__HIP_PLATFORM_AMD__", "-DUSE_ROCM",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}", "-I", INCLUDE,
           *[f"-isystem{d}" for d in system], "-c", src, "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"compiling {src} failed:\n{r.stdout}{r.stderr}")
    return obj, r.stdout + r.stderr


def _link(name, to, cmd):
    tmp = to + ".tmp"
    r = subprocess.run([*cmd, "-o", tmp], capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"linking {name} failed:\n{r.stdout}{r.stderr}")
    os.replace(tmp, to)


def build(verbose=False):
    import torch
    os.makedirs(OBJDIR, exist_ok=True)
    with concurrent.futures.ThreadPoolExecutor(max_workers=min(8, os.cpu_count() or 1)) as ex:
        pending = ex.submit(_compile_binding)
        results = list(ex.map(_compile, sources()))
        binding = pending.result()
    for _, msgs in (*results, binding):
        if verbose and msgs.strip():
            print(msgs, file=sys.stderr)
    _link("libwavezip.so", LIB, [hipcc(), "-shared", f"--offload-arch={ARCH}", *[o for o, _ in results]])
    libs = os.path.join(os.path.dirname(torch.__file__), "lib")
    _link("_serve.so", BINDING, ["g++", "-shared", binding[0], "-L", PKG, "-l:libwavezip.so", "-L", libs, "-ltorch_python",
                                 "-ltorch_cpu", "-lc10_hip", "-lc10", "-Wl,-rpath,$ORIGIN"])
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
