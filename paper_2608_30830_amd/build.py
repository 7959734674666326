"""Build libkvr.so for gfx950 with hipcc, and its binding to torch tensors (in-tree, under
``_build/``)."""
from __future__ import annotations

import concurrent.futures as cf
import os
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
OUT_DIR = os.path.join(PKG, "_build")
LIB = os.path.join(OUT_DIR, "libkvr.so")
BINDING = os.path.join(OUT_DIR, "kvr_torch.so")   # host code on torch tensors, over libkvr
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
ROCM = os.path.dirname(os.path.dirname(HIPCC)) if os.path.isabs(HIPCC) else "/opt/rocm"
CXX = os.environ.get("CXX", "g++")

SOURCES = ["kvr_api.cpp", "kvr_grid.hip", "kvr_aux.hip", "kvr_sorted.hip", "kvr_binned.hip",
           "kvr_replay.hip",
           "kvr_controller.hip", "kvr_r3.hip",
           "kvr_factored.hip", "kvr_noalloc.hip", "kvr_small.hip",
           "kvr_kv_api.cpp", "kvr_rotary.hip", "kvr_cache.hip", "kvr_attention.hip",
           "kvr_attention_bf16.hip", "kvr_attention_fp16.hip", "kvr_attention_fp8.hip",
           "kvr_attention_fp8h.hip", "kvr_attention_fp4.hip", "kvr_attention_fp4h.hip",
           "kvr_latent_api.cpp", "kvr_latent.hip", "kvr_latent_cache.hip", "kvr_latent_bf16.hip",
           "kvr_latent_fp16.hip", "kvr_latent_fp8.hip", "kvr_prompt.hip",
           "kvr_pages_api.cpp", "kvr_pages.hip"]
# Kernels that meet whatever a model or unwritten memory holds: NaNs are kept.
NAN_SAFE = tuple(s for s in SOURCES if s.startswith(("kvr_rotary", "kvr_cache", "kvr_attention",
                                                     "kvr_latent", "kvr_prompt")))
# Kernels whose accumulators are more than 256 registers: matrix instructions may then take
# them from either half of the register file (else hundreds of registers go to memory).
WIDE = ("kvr_latent_bf16.hip", "kvr_latent_fp16.hip", "kvr_latent_fp8.hip", "kvr_prompt.hip")
COMMON = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
          # no packed-fp32 instruction selection anywhere
          "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
          "-I" + os.path.join(ROOT, "include"), "-I" + CSRC]
# Device code only (but NAN_SAFE): every sample is validated on its bits before use and no
# NaN ever reaches the arithmetic, so min/max need no NaN quieting.
DEVICE = ["-Xarch_device", "-fno-honor-nans"]


def _compile(src: str) -> str:
    obj = os.path.join(OUT_DIR, os.path.basename(src) + ".o")
    cmd = [HIPCC] + COMMON + (DEVICE if src.endswith(".hip") and src not in NAN_SAFE else []) + \
        (["-mllvm", "-amdgpu-mfma-vgpr-form=1"] if src in WIDE else []) + \
        ["-c", os.path.join(CSRC, src), "-o", obj]
    subprocess.run(cmd, check=True, stdout=subprocess.PIPE, stderr=subprocess.STDOUT)
    return obj


def _compile_binding() -> str:
    import sysconfig
    import torch
    root = os.path.dirname(torch.__file__)
    obj = os.path.join(OUT_DIR, "kvr_torch.cpp.o")
    includes = [os.path.join(root, "include"), os.path.join(root, "include/torch/csrc/api/include"),
                sysconfig.get_paths()["include"], os.path.join(ROCM, "include"),
                os.path.join(ROOT, "include")]
    cmd = [CXX, "-O2", "-std=c++17", "-fPIC", "-DUSE_ROCM", "-D__HIP_PLATFORM_AMD__=1",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}"]
    cmd += [x for i in includes for x in ("-isystem", i)]
    subprocess.run(cmd + ["-c", os.path.join(CSRC, "kvr_torch.cpp"), "-o", obj], check=True,
                   stdout=subprocess.PIPE, stderr=subprocess.STDOUT)
    return obj


def _link_binding(obj: str) -> None:
    import torch
    libs = os.path.join(os.path.dirname(torch.__file__), "lib")
    tmp = BINDING + f".tmp{os.getpid()}"
    subprocess.run([CXX, "-shared", "-fPIC", "-o", tmp, obj, LIB, "-L" + libs, "-ltorch_python",
                    "-ltorch", "-ltorch_cpu", "-lc10", "-lc10_hip",
                    "-Wl,-rpath,$ORIGIN", "-Wl,-rpath," + libs],
                   check=True, stdout=subprocess.PIPE, stderr=subprocess.STDOUT)
    os.replace(tmp, BINDING)


def build(verbose: bool = False) -> str:
    """Compile every source, link libkvr.so and the binding; always rebuilds."""
    os.makedirs(OUT_DIR, exist_ok=True)
    try:
        with cf.ThreadPoolExecutor(max_workers=len(SOURCES) + 1) as ex:
            binding = ex.submit(_compile_binding)
            objs = list(ex.map(_compile, SOURCES))
            binding = binding.result()
        tmp = LIB + f".tmp{os.getpid()}"
        subprocess.run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-Wl,-soname,libkvr.so",
                        "-o", tmp] + objs,
                       check=True, stdout=subprocess.PIPE, stderr=subprocess.STDOUT)
        os.replace(tmp, LIB)
        _link_binding(binding)
    except subprocess.CalledProcessError as err:
        sys.stderr.write(err.stdout.decode(errors="replace"))
        raise
    if verbose:
        print(f"built {LIB}")
    return LIB


if __name__ == "__main__":
    build(verbose=True)
