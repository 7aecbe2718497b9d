"""Builds libesp_hip.so (gfx950) in-tree with hipcc.  `python -m paper_2603_17942_amd.build`."""
from __future__ import annotations

import concurrent.futures
import os
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libesp_hip.so")
SOURCES = ["esp_api.hip", "esp_elementwise.hip", "esp_gemm.hip", "esp_gemm_tile_out.hip", "esp_gemm_tile_argmax.hip",
           "esp_gemm_tile_swiglu.hip", "esp_gemm_tile_both.hip", "esp_attn.hip", "esp_topk.hip", "esp_tree.hip",
           "esp_paged_api.hip", "esp_paged.hip", "esp_paged_attn.hip", "esp_sample.hip", "esp_paged_weigh.hip", "esp_paged_evict.hip"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-I" + os.path.join(ROOT, "include"),
         "-I" + CSRC, "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-Wno-unused-command-line-argument"]


# per-source additions: the attention kernels never produce or test NaN / infinity (masked scores are a
# large finite negative), and telling the compiler so drops the canonicalising copy in front of
# every maximum of the online softmax; the scores of the paged attention and of the attention weights are wanted in VGPRs,
# where their softmax reads them, also in kernels with more than 256 registers
EXTRA_FLAGS = {"esp_attn.hip": ["-fno-honor-nans"], "esp_paged_attn.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form=1"],
               "esp_paged_weigh.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form=1"]}


def _compile(src: str) -> str:
    obj = os.path.join(PKG, "_build", src.replace(".hip", ".o"))
    os.makedirs(os.path.dirname(obj), exist_ok=True)
    cmd = [HIPCC, *FLAGS, *EXTRA_FLAGS.get(src, []), "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed on {src}:\n{r.stdout}\n{r.stderr}")
    noise = "is not a recognized feature for this target"
    err = "\n".join(l for l in r.stderr.splitlines() if noise not in l)
    if err.strip():
        sys.stderr.write(err + "\n")
    return obj


def build(verbose: bool = True) -> str:
    with concurrent.futures.ThreadPoolExecutor(max_workers=8) as ex:
        objs = list(ex.map(_compile, SOURCES))
    r = subprocess.run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", *objs, "-o", LIB],
                       capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
    if verbose:
        print("built", LIB)
    return LIB


if __name__ == "__main__":
    build()
