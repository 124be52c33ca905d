"""Build libbagel.so (HIP, gfx950) in-tree with hipcc, and _marshal.so (the binding's checks of torch tensors) with g++.
``python -m paper_2202_13638_amd.build``."""
from __future__ import annotations

import concurrent.futures as cf
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libbagel.so")
MARSHAL = os.path.join(HERE, "_marshal.so")
SOURCES = ["adamw.hip", "backward.hip", "bagel_api.hip", "block_join.hip", "clip.hip", "gp_step.hip", "lane.hip", "layer_norm.hip", "model.hip", "policy.hip", "policy16.hip", "posterior.hip", "prepare.hip", "recurrence.hip", "rollout.hip"]
# linear attention: what has matrix instructions of 16-bit operands, whose results are waited for by other rules (tests/test_more_matrix_wait_states.py)
MATRIX_16_SOURCES = ["linear_attention.hip", "linear_attention_bf16.hip", "linear_attention_f16.hip", "linear_attention_f32.hip"]
# -packed-fp32-ops is switched off on purpose: no packed float32 VALU instructions in this library
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-ffp-contract=off",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-Wall", "-Wno-unused-function"]


def _compile(src: str, force: bool) -> str:
    obj = os.path.join(BUILD, src.replace(".hip", ".o"))
    path = os.path.join(CSRC, src)
    deps = [path, *(os.path.join(CSRC, h) for h in os.listdir(CSRC) if h.endswith(".h")),
            os.path.join(ROOT, "include", "bagel.h"), __file__]
    if not force and os.path.exists(obj) and all(os.path.getmtime(obj) >= os.path.getmtime(d) for d in deps):
        return obj
    cmd = ["hipcc", *FLAGS, "-c", path, "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed for {src}:\n{r.stdout}\n{r.stderr}")
    warn = [ln for ln in r.stderr.splitlines() if "packed-fp32-ops" not in ln and ln.strip()]
    if warn:
        sys.stderr.write("\n".join(warn) + "\n")
    return obj


def _marshal(force: bool) -> None:
    import sysconfig
    import torch
    from torch.utils import cpp_extension
    path, header = os.path.join(CSRC, "marshal.cpp"), os.path.join(ROOT, "include", "bagel.h")
    if not force and os.path.exists(MARSHAL) and all(os.path.getmtime(MARSHAL) >= os.path.getmtime(d) for d in (path, header, __file__)):
        return
    lib = os.path.join(os.path.dirname(torch.__file__), "lib")
    cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           "-I", os.path.join(ROOT, "include"), "-I", sysconfig.get_path("include"),
           *(f for d in cpp_extension.include_paths() if "torch" in d for f in ("-isystem", d)), path, "-o", MARSHAL,
           "-L", lib, "-ltorch_python", "-ltorch_cpu", "-lc10"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"g++ failed for marshal.cpp:\n{r.stdout}\n{r.stderr}")


def build(force: bool = False) -> str:
    os.makedirs(BUILD, exist_ok=True)
    with cf.ThreadPoolExecutor(max_workers=6) as ex:
        marshal = ex.submit(_marshal, force)
        objs = list(ex.map(lambda s: _compile(s, force), MATRIX_16_SOURCES + SOURCES))
        marshal.result()
    if force or not os.path.exists(LIB) or any(os.path.getmtime(o) > os.path.getmtime(LIB) for o in objs):
        cmd = ["hipcc", "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB, *objs]
        subprocess.run(cmd, check=True)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv))
