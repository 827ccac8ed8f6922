"""Compiles the HIP sources into paper_2201_05596_amd/libmoe_hip.so for gfx950.

hipcc cross-compiles without a GPU.  Usage: ``python -m paper_2201_05596_amd.build``.
"""
from __future__ import annotations

import os
import re
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libmoe_hip.so")
SOURCES = ["api.hip", "gate.hip", "gate_bf16.hip", "layout.hip", "pack.hip", "block.hip", "rope.hip", "kv_cache.hip", "tree_attn.hip", "tree_attn_bf16.hip", "tree_attn_fp8.hip", "tree_attn_fp4.hip", "i8_quant.hip", "i8_few.hip", "i8_token.hip", "i8_tile.hip", "i8_wide.hip", "gemm_f32.hip", "ffn_mfma.hip", "ffn_rows.hip", "ffn_tile.hip", "ffn_wide.hip",
           "ffn_wide_store.hip", "ffn_wide_gelu.hip", "ffn_wide_scatter.hip"]

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-fno-gpu-rdc",
    # keep the compiler from forming packed-fp32 instructions
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wno-unused-command-line-argument",
    "-I", os.path.join(ROOT, "include"), "-I", CSRC,
]


# Sources whose kernels must keep nothing in scratch memory: a build that does not is refused.  (Not among them: the tiles of 256 rows, ffn_wide*.hip and
# i8_wide.hip, which take every register; some keep up to three of the epilogue's values there, outside of the main loop.)
NO_SCRATCH = ("tree_attn_bf16.hip", "tree_attn_fp8.hip", "tree_attn_fp4.hip", "i8_quant.hip", "i8_few.hip", "i8_token.hip", "i8_tile.hip")


def kernels_in_scratch(remarks: str) -> list:
    """Names of the kernels that the compiler's remarks on resource usage say have values in scratch memory."""
    sizes = re.findall(r"Function Name: (\S+).*?ScratchSize \[bytes/lane\]: (\d+)", remarks, re.S)
    if not sizes:
        raise RuntimeError("the compiler says nothing on resource usage")
    return [name for name, size in sizes if int(size)]


def _compile(src: str) -> str:
    obj_dir = os.path.join(HERE, "_build")
    os.makedirs(obj_dir, exist_ok=True)
    obj = os.path.join(obj_dir, src.replace(".hip", ".o"))
    cmd = [HIPCC, *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
    if src in NO_SCRATCH:
        cmd.append("-Rpass-analysis=kernel-resource-usage")
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed for {src}:\n{r.stdout}\n{r.stderr}")
    if src in NO_SCRATCH and (bad := kernels_in_scratch(r.stderr)):
        os.remove(obj)
        raise RuntimeError(f"{src}: values in scratch memory: {', '.join(bad)}")
    return obj


def build(verbose: bool = True) -> str:
    with ThreadPoolExecutor(max_workers=min(8, len(SOURCES))) as ex:
        objs = list(ex.map(_compile, SOURCES))
    cmd = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB, *objs,
           "-Wl,-rpath,/opt/rocm/lib", "-Wl,-soname,libmoe_hip.so"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
    if verbose:
        print(f"built {LIB}")
    return LIB


if __name__ == "__main__":
    build()
    sys.exit(0)
