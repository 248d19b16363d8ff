"""Compile the HIP kernels and the C-ABI runtime into ``libvlaprefix.so``
(gfx950 only) with hipcc, and the binding's torch calls of the 4-bit and 8-bit operators
into ``_torch_ops.so``.  Objects go to ``_build/`` next to this file."""
from __future__ import annotations

import concurrent.futures as cf
import importlib.util
import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OUT_DIR = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libvlaprefix.so")
TORCH_OPS = os.path.join(HERE, "_torch_ops.so")

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
ARCH = "gfx950"
# Packed-fp32 VALU ops are switched off for all device code.
DEVICE_FLAGS = ["--offload-arch=" + ARCH, "-O3", "-fPIC", "-std=c++17", "-Xclang", "-target-feature", "-Xclang",
                "-packed-fp32-ops", "-Wno-unused-result"]
HOST_FLAGS = ["-O2", "-fPIC", "-std=c++17", "-Wall", "-Wno-unused-result"]

SOURCES = ["gemm_bf16.hip", "attention_bf16.hip", "decode_bf16.hip", "norm.hip", "fp32_path.hip", "vision.hip",
           "static_scratch.hip", "w4.hip", "qk_norm.hip", "kv4.hip", "norm_i8.hip", "w8.hip", "kv8.hip", "attention_packed.hip",
           "runtime.cpp",
           "ops.cpp",
           "host_suffix.cpp", "host_suffix_api.cpp", "sched.cpp"]
# Attention keeps its score and output accumulators in VGPRs: the softmax
# touches them every key tile, and AGPR accumulators would cost a copy each way.
EXTRA = {"attention_bf16.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"],
         "attention_packed.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"],
         # the results of their MFMAs are scaled right after them
         "kv4.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"], "w4.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"],
         "kv8.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form"],
         # the host suffix executor: AVX-512 BF16 kernels, entered only after a CPU check
         "host_suffix.cpp": ["--offload-host-only", "-O3", "-mavx512f", "-mavx512bw", "-mavx512vl", "-mavx512bf16",
                             "-mfma"],
         "host_suffix_api.cpp": ["--offload-host-only"],
         "sched.cpp": ["--offload-host-only"]}


def _compile(src: str) -> str:
    path = os.path.join(CSRC, src)
    obj = os.path.join(OUT_DIR, src + ".o")
    if src.endswith(".hip"):
        cmd = [HIPCC] + DEVICE_FLAGS + EXTRA.get(src, []) + ["-c", path, "-o", obj]
    else:
        cmd = [HIPCC] + HOST_FLAGS + EXTRA.get(src, []) + ["-c", path, "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("hipcc failed for %s:\n%s\n%s" % (src, " ".join(cmd), r.stderr[-6000:]))
    return obj


def _torch_dir() -> str:
    spec = importlib.util.find_spec("torch")
    if spec is None:
        raise RuntimeError("_torch_ops.so, the 4-bit and 8-bit operators on torch tensors, needs torch's headers and libraries, "
                           "and torch is not installed (libvlaprefix.so does without)")
    return list(spec.submodule_search_locations)[0]


def _compile_torch_ops() -> str:
    """Host code only: torch tensors in, calls of the C ABI out."""
    obj = os.path.join(OUT_DIR, "torch_ops.cpp.o")
    inc = os.path.join(_torch_dir(), "include")
    cmd = ["g++", "-D__HIP_PLATFORM_AMD__"] + HOST_FLAGS + \
        ["-I" + d for d in (inc, os.path.join(inc, "torch", "csrc", "api", "include"), "/opt/rocm/include",
                            sysconfig.get_paths()["include"])] + ["-c", os.path.join(CSRC, "torch_ops.cpp"), "-o", obj]
    try:
        r = subprocess.run(cmd, capture_output=True, text=True)
    except FileNotFoundError:
        raise RuntimeError("_torch_ops.so, the 4-bit and 8-bit operators on torch tensors, needs g++ (libvlaprefix.so does without)")
    if r.returncode != 0:
        raise RuntimeError("g++ failed for torch_ops.cpp:\n%s\n%s" % (" ".join(cmd), r.stderr[-6000:]))
    return obj


def _link(cmd, out: str) -> None:
    tmp = out + ".tmp%d" % os.getpid()
    r = subprocess.run(cmd + ["-o", tmp], capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed:\n%s\n%s" % (" ".join(cmd), r.stderr[-4000:]))
    os.replace(tmp, out)


def build(verbose: bool = False) -> str:
    """Compile every source and link the shared library, then the module of torch
    calls (where that cannot be built the library is there all the same);
    returns the library's path."""
    os.makedirs(OUT_DIR, exist_ok=True)
    with cf.ThreadPoolExecutor(max_workers=min(8, len(SOURCES) + 1)) as ex:
        torch_obj = ex.submit(_compile_torch_ops)
        objs = list(ex.map(_compile, SOURCES))
    _link([HIPCC, "--offload-arch=" + ARCH, "-shared", "-fPIC"] + objs, LIB)
    _link(["g++", "-shared", torch_obj.result(), "-L" + HERE, "-lvlaprefix", "-Wl,-rpath,$ORIGIN",
           "-L" + os.path.join(_torch_dir(), "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10_hip", "-lc10"], TORCH_OPS)
    if verbose:
        print("built", LIB)
    return LIB


if __name__ == "__main__":
    build(verbose=True)
    sys.exit(0)
