"""Compile the HIP sources under csrc/ into paper_2302_14357_amd/libtbs.so for gfx950."""

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libtbs.so")
BINDING = os.path.join(HERE, "_tbs_ops.so")
SOURCES = ["tbs_api.hip", "beam_kernels.hip", "expand_kernels.hip", "joiner_kernels.hip", "gemm_kernels.hip", "gemm_f32_kernels.hip", "pred_kernels.hip", "round_kernels.hip", "xcd_kernels.hip", "xcd_f32_kernels.hip", "xcd_long_kernels.hip", "xcd_push_kernels.hip",
           "linear_kernels.hip", "linear_f16_kernels.hip", "linear_f32_kernels.hip", "attend_kernels.hip", "vocab_kernels.hip", "pages_kernels.hip"]
FLAGS = ["-O3", "-std=c++17", "--offload-arch=gfx950", "-fPIC", "-fno-gpu-rdc",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-Wall", "-Wno-unused-result"]


def binding_command() -> list:
    """The host compiler's call for the Python module of the operators (csrc/ops_binding.cpp): torch's tensors in, calls of libtbs out."""
    import sysconfig
    import torch
    t = os.path.dirname(torch.__file__)
    inc = [sysconfig.get_paths()["include"], os.path.join(t, "include"), os.path.join(t, "include", "torch", "csrc", "api", "include"), "/opt/rocm/include",
           os.path.join(ROOT, "include")]
    return ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-D__HIP_PLATFORM_AMD__=1", "-DUSE_ROCM=1", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}",
            *[f"-I{i}" for i in inc], os.path.join(CSRC, "ops_binding.cpp"), "-o", BINDING, f"-L{HERE}", "-l:libtbs.so", f"-L{os.path.join(t, 'lib')}", "-lc10", "-lc10_hip",
            "-ltorch_cpu", "-ltorch_python", "-Wl,-rpath,$ORIGIN"]


def build(verbose: bool = False) -> str:
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    objs = []
    procs = []
    for s in SOURCES:
        o = os.path.join(CSRC, s.replace(".hip", ".o"))
        objs.append(o)
        cmd = [hipcc, *FLAGS, "-c", os.path.join(CSRC, s), "-o", o]
        procs.append((cmd, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    for cmd, p in procs:
        out, _ = p.communicate()
        out = "\n".join(l for l in out.splitlines() if "packed-fp32-ops" not in l)
        if p.returncode != 0:
            raise RuntimeError("hipcc failed: " + " ".join(cmd) + "\n" + out)
        if verbose and out.strip():
            print(out)
    cmd = [hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB, *objs]
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed:\n" + r.stdout)
    cmd = binding_command()
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    if r.returncode != 0:
        raise RuntimeError("g++ failed: " + " ".join(cmd) + "\n" + r.stdout)
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
    sys.exit(0)
