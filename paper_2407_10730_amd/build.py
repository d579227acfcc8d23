"""Build the gfx950 conv2d library (libconv2d.so) in-tree with hipcc."""
import concurrent.futures as cf
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libconv2d.so")
HARNESS = os.path.join(HERE, "convbench")
PYCALL = os.path.join(HERE, "_seqmix.so")
SOURCES = ["conv2d_api.hip", "gemm_mfma.hip", "pack_kernels.hip", "direct_kernels.hip", "slice_conv.hip",
           "probes.hip", "winograd.hip", "patch_conv.hip", "seqmix_api.hip", "linattn.hip",
           "linattn_chunks.hip", "linattn_chunks_f32.hip", "token_conv.hip", "gate_norm.hip"]

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    # never let the compiler form packed-fp32 VALU ops
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-result",
    "-I" + os.path.join(ROOT, "include"), "-I" + CSRC,
]


def _compile(src, verbose):
    obj = os.path.join(BUILD, os.path.splitext(src)[0] + ".o")
    cmd = [HIPCC, *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, capture_output=True, text=True)
    out = "\n".join(l for l in (r.stdout + r.stderr).splitlines()
                    if "packed-fp32-ops" not in l and "is not a recognized feature" not in l)
    return src, r.returncode, out, obj


def _build_pycall(verbose):
    """The Python side of seqmix.py's calls (host code against the installed torch)."""
    import sysconfig

    import torch
    from torch.utils import cpp_extension as ce
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           *["-I" + p for p in ce.include_paths()], "-I" + sysconfig.get_paths()["include"],
           os.path.join(CSRC, "seqmix_py.cpp"), *["-L" + p for p in ce.library_paths()[:1]],
           "-ltorch_python", "-ltorch_cpu", "-lc10", "-o", PYCALL + ".tmp"]
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        print(r.stdout + r.stderr, file=sys.stderr)
        raise RuntimeError("g++ failed for seqmix_py.cpp")
    os.replace(PYCALL + ".tmp", PYCALL)


def build(verbose: bool = False) -> str:
    os.makedirs(BUILD, exist_ok=True)
    with cf.ThreadPoolExecutor(max_workers=min(8, len(SOURCES))) as ex:
        results = list(ex.map(lambda s: _compile(s, verbose), SOURCES))
    failed = [r for r in results if r[1] != 0]
    for src, rc, out, _ in results:
        if out.strip() and (verbose or rc != 0):
            print(f"--- {src}\n{out}", file=sys.stderr)
    if failed:
        raise RuntimeError("hipcc failed for: " + ", ".join(r[0] for r in failed))
    tmp = LIB + ".tmp"
    cmd = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", *[r[3] for r in results], "-o", tmp]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)
    os.replace(tmp, LIB)
    # the ConvBench-style harness (host code over the library's C ABI)
    tmp = HARNESS + ".tmp"
    cmd = [HIPCC, "-O2", "-std=c++17", "-Wall", "-I" + os.path.join(ROOT, "include"),
           os.path.join(CSRC, "convbench.cpp"), "-o", tmp, "-L" + HERE, "-lconv2d", "-Wl,-rpath,$ORIGIN"]
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        print(r.stdout + r.stderr, file=sys.stderr)
        raise RuntimeError("hipcc failed for convbench.cpp")
    os.replace(tmp, HARNESS)
    _build_pycall(verbose)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
