"""Builds libnetmax.so (HIP, gfx950) in-tree with hipcc, and the extension module of the calls on torch's tensors with g++."""
from __future__ import annotations

import importlib.util
import os
import subprocess
import sysconfig
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(PKG, "csrc")
OBJ = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libnetmax.so")
CALLS = os.path.join(PKG, "_lm_calls.so")              # extension module: calls on torch's tensors

SOURCES = ["netmax_api.hip", "k_small_iter.hip", "k_sliced_iter.hip", "k_resident_mlp.hip", "k_sample.hip", "k_synth_grad.hip", "k_mix.hip", "k_consensus.hip", "k_grad_mlp.hip",
           "k_layout.hip", "k_grad_mfma.hip", "k_grad_head.hip", "k_grad_f32.hip", "policy.hip", "k_async.hip", "k_mix_subset.hip", "k_mix_synth.hip",
           "k_tile_fwd.hip", "k_tile_dgrad.hip", "k_tile_wgrad.hip", "k_chain.hip",
           "lm_api.hip", "k_linear.hip", "k_orth.hip", "k_token_loss.hip",
           "lm_step_api.hip", "k_embed.hip", "k_block_norm.hip", "k_clip.hip"]

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Wall", "-Wno-unused-result",
         # packed fp32 instructions are kept out of the generated code
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]


def _compile(src: str) -> str:
    obj = os.path.join(OBJ, src.replace(".hip", ".o"))
    subprocess.run([HIPCC, *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj], check=True)
    return obj


def build_calls() -> str:
    torch = os.path.dirname(importlib.util.find_spec("torch").origin)
    include = [os.path.join(torch, "include"), os.path.join(torch, "include", "torch", "csrc", "api", "include"), sysconfig.get_paths()["include"]]
    subprocess.run(["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", "-Wno-cast-function-type", *(f"-isystem{d}" for d in include), os.path.join(CSRC, "lm_calls.cpp"), "-o", CALLS,
                    "-L" + os.path.join(torch, "lib"), "-lc10", "-ltorch_cpu", "-ltorch_python"], check=True)
    return CALLS


def build(verbose: bool = False) -> str:
    os.makedirs(OBJ, exist_ok=True)
    with ThreadPoolExecutor(max_workers=min(8, len(SOURCES))) as ex:
        calls = ex.submit(build_calls)
        objs = list(ex.map(_compile, SOURCES))
        calls.result()
    subprocess.run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB, *objs], check=True)
    if verbose:
        print("built", LIB)
    return LIB


if __name__ == "__main__":
    build(verbose=True)
