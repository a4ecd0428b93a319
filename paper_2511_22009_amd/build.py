"""Build libstreamflow.so (all HIP kernels + the C-ABI runtime) for gfx950, in-tree, and the
binding of the operators on torch tensors.

    python -m paper_2511_22009_amd.build

Objects go to <repo>/_build/; the libraries are written next to this file.
"""
import concurrent.futures
import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
OUT = os.path.join(HERE, "libstreamflow.so")
BUILD_DIR = os.path.join(ROOT, "_build")
SOURCES = ["k_cond.hip", "k_norm.hip", "k_gemm.hip", "k_attn.hip", "k_euler.hip", "k_quant.hip",
           "k_gemm_i8.hip", "k_rope.hip", "streamflow.cpp", "operators.cpp"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
CXX = os.environ.get("CXX", "g++")
ARCH = "gfx950"
FLAGS = ["-O3", "-std=c++17", "-fPIC", f"--offload-arch={ARCH}",
         # keep the compiler from emitting packed-fp32 VALU instructions
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-I", INCLUDE, "-I", CSRC]
# Per-source flags. Attention runs VALU softmax work on the MFMA results (scores and
# the running output), so their accumulators are kept in architectural VGPRs instead
# of being copied to and from accumulation registers every key block.
SOURCE_FLAGS = {"k_attn.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form=1"]}


def _compile(src):
    obj = os.path.join(BUILD_DIR, os.path.splitext(src)[0] + ".o")
    cmd = [HIPCC, *FLAGS, *SOURCE_FLAGS.get(src, []), "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    msgs = "\n".join(l for l in (r.stdout + r.stderr).splitlines() if "packed-fp32-ops" not in l)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed on {src}:\n{msgs}")
    return obj, msgs


def _build_operators():
    """The binding of the operators: host code against torch's headers, no HIP in it."""
    import torch
    from torch.utils.cpp_extension import include_paths
    lib = os.path.join(os.path.dirname(torch.__file__), "lib")
    out = os.path.join(HERE, "_operators" + sysconfig.get_config_var("EXT_SUFFIX"))
    tmp = out + ".tmp"
    cmd = [CXX, "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden", "-Wall",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           "-I", INCLUDE, *[f for p in (*include_paths(), sysconfig.get_paths()["include"]) for f in ("-isystem", p)],
           os.path.join(CSRC, "py_operators.cpp"), "-o", tmp, "-L", lib, "-lc10", "-ltorch_cpu", "-ltorch_python"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"{CXX} failed on py_operators.cpp:\n{r.stdout}{r.stderr}")
    os.replace(tmp, out)
    return r.stdout + r.stderr


def build(verbose=False):
    os.makedirs(BUILD_DIR, exist_ok=True)
    with concurrent.futures.ThreadPoolExecutor(max_workers=min(8, len(SOURCES) + 1)) as ex:
        binding = ex.submit(_build_operators)
        results = list(ex.map(_compile, SOURCES))
        results.append((None, binding.result()))
    if verbose:
        for _, msgs in results:
            if msgs.strip():
                print(msgs)
    tmp = OUT + ".tmp"
    cmd = [HIPCC, "-shared", "-fPIC", f"--offload-arch={ARCH}", *[o for o, _ in results if o], "-o", tmp]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}{r.stderr}")
    os.replace(tmp, OUT)
    return OUT


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
