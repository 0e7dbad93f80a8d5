"""Build libmiconv.so (the HIP kernels and the C ABI), _mitrain.so (the Python
binding of include/mitrain.h and include/mistep.h) and libmipeak.so (the benchmark's measured
reference points) in-tree for gfx950."""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

if __package__ in (None, ""):
    sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIBRARY = os.path.join(PKG, "libmiconv.so")
SOURCES = ["api.hip", "conv_kernels.hip", "wino_kernels.hip", "pool_kernels.hip",
           "train_api.hip", "norm_kernels.hip", "logprob_kernels.hip", "clip_kernels.hip",
           "step_api.hip", "dropout_kernels.hip", "residual_kernels.hip", "loss_kernels.hip"]
PEAK_LIBRARY = os.path.join(PKG, "libmipeak.so")
PEAK_SOURCES = ["peaks.hip"]
BINDING = os.path.join(PKG, "_mitrain.so")
BINDING_SOURCES = ["binding.cpp", "binding_step.cpp"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
    "-Wall", "-Wno-unused-result",
    # Keep the compiler from forming packed fp32 VALU ops.
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-I", os.path.join(ROOT, "include"),
]


def _hipcc(args, verbose):
    _run([HIPCC] + args, verbose)


def _run(cmd, verbose):
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    # hipcc's host pass warns that it does not know the packed-fp32 feature.
    text = "\n".join(l for l in res.stdout.splitlines()
                     if "packed-fp32-ops' is not a recognized feature" not in l)
    if res.returncode != 0:
        raise RuntimeError(f"{cmd[0]} failed ({res.returncode}):\n{text}")
    if text.strip() and verbose:
        print(text, file=sys.stderr)


def _compile(sources, out, verbose):
    """Each source to an object (several at a time), the objects to out.tmp."""
    tmp = out + ".tmp"
    flags = [f for f in FLAGS if f != "-shared"]
    with tempfile.TemporaryDirectory() as obj_dir, ThreadPoolExecutor(4) as pool:
        objs = [os.path.join(obj_dir, s + ".o") for s in sources]
        list(pool.map(lambda so: _hipcc(
            flags + ["-c", os.path.join(CSRC, so[0]), "-o", so[1]], verbose),
            zip(sources, objs)))
        _hipcc(["--offload-arch=gfx950", "-fPIC", "-shared"] + objs + ["-o", tmp], verbose)
    return tmp


def _binding(verbose):
    """The binding is host code on torch's headers: no HIP compiler."""
    import sysconfig

    import torch
    lib = os.path.join(os.path.dirname(torch.__file__), "lib")
    include = os.path.join(os.path.dirname(torch.__file__), "include")
    tmp = BINDING + ".tmp"
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-fvisibility=hidden", "-Wall",
           "-D__HIP_PLATFORM_AMD__=1", "-DUSE_ROCM=1",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           "-I", os.path.join(ROOT, "include"),
           "-isystem", include, "-isystem", os.path.join(include, "torch", "csrc", "api", "include"),
           "-isystem", sysconfig.get_paths()["include"],
           "-isystem", os.path.join(os.path.dirname(os.path.dirname(HIPCC)), "include")]
    with tempfile.TemporaryDirectory() as obj_dir, ThreadPoolExecutor(2) as pool:
        objs = [os.path.join(obj_dir, s + ".o") for s in BINDING_SOURCES]
        list(pool.map(lambda so: _run(
            cmd + ["-c", os.path.join(CSRC, so[0]), "-o", so[1]], verbose),
            zip(BINDING_SOURCES, objs)))
        _run(["g++", "-shared"] + objs + ["-o", tmp, "-L", lib, "-lc10", "-lc10_hip",
                                          "-ltorch_cpu", "-ltorch_python"], verbose)
    return tmp


def build(verbose: bool = False) -> str:
    tmp = _compile(SOURCES, LIBRARY, verbose)
    # The image GEMM's untracked filter loads are only correct if the
    # compiler kept their registers out of reach while in flight.
    from paper_1903_06934_amd import isa_check
    isa_check.check(HIPCC, FLAGS, os.path.join(CSRC, "conv_kernels.hip"))
    os.replace(tmp, LIBRARY)
    os.replace(_compile(PEAK_SOURCES, PEAK_LIBRARY, verbose), PEAK_LIBRARY)
    # Last, as it alone needs torch's headers and a host compiler.
    os.replace(_binding(verbose), BINDING)
    return LIBRARY


if __name__ == "__main__":
    print(build(verbose=True))
