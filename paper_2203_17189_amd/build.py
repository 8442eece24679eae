"""Compile the HIP sources of this package into libt5mi.so for gfx950 (in-tree, beside this file)."""
from __future__ import annotations

import os
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libt5mi.so")
OBJ_DIR = os.path.join(HERE, "_build")
SOURCES = ["relpos.hip", "rmsnorm.hip", "gemm_simple.hip", "gemm_mfma.hip", "gemm_mfma_store.hip",
           "gemm_mfma_resid.hip", "gemm_mfma_geglu_fwd.hip", "gemm_mfma_geglu_bwd.hip", "gemm_mfma_split.hip",
           "gemm_mfma_split_grouped.hip", "gemm_mfma_direct.hip", "gemm_f32.hip", "attn_simple.hip",
           "attn_mfma.hip", "attn_f32.hip", "adafactor.hip", "probe.hip", "embed_xent.hip", "embed_sorted.hip", "top_logits.hip", "distill.hip",
           "quant_fp8.hip", "gemm_fp8.hip", "gemm_fp8_44.hip", "gemm_fp8_45.hip", "gemm_fp8_54.hip", "gemm_fp8_55.hip", "gemm_fp8_rows.hip", "adamw.hip",
           "block.hip", "stack.hip", "vocab_ops.hip", "fp8_ops.hip"]
# -packed-fp32-ops is switched off: hand-written and compiler-made packed float32 math is avoided on
# this target.
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Xclang", "-target-feature", "-Xclang",
         "-packed-fp32-ops", "-Wno-unused-command-line-argument"]


LISTS = os.path.join(HERE, "_torch_lists" + sysconfig.get_config_var("EXT_SUFFIX"))


def build_lists() -> str:
    """The Python module that reads lists of tensors (host code only, against torch's headers)."""
    import torch
    root = os.path.dirname(torch.__file__)
    inc = [sysconfig.get_paths()["include"], os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include")]
    lib = os.path.join(root, "lib")
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           *[f"-I{i}" for i in inc], os.path.join(CSRC, "torch_lists.cpp"), "-o", LISTS, f"-L{lib}", "-ltorch_python", "-ltorch_cpu", "-lc10",
           f"-Wl,-rpath,{lib}"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"g++ failed for torch_lists.cpp:\n{r.stdout}\n{r.stderr}")
    return LISTS


def _compile(src: str) -> str:
    obj = os.path.join(OBJ_DIR, src.replace(".hip", ".o"))
    cmd = ["hipcc", *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed for {src}:\n{r.stdout}\n{r.stderr}")
    return obj


def build(verbose: bool = True) -> str:
    os.makedirs(OBJ_DIR, exist_ok=True)
    with ThreadPoolExecutor(max_workers=min(8, len(SOURCES))) as ex:
        lists = ex.submit(build_lists)
        objs = list(ex.map(_compile, SOURCES))
    lists.result()
    cmd = ["hipcc", "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB, *objs]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
    if verbose:
        print(f"built {LIB}")
    return LIB


if __name__ == "__main__":
    build()
    sys.exit(0)
