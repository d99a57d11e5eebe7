"""Build libkvk.so for gfx950 in-tree with hipcc.

Usage: python -m paper_2609_37988_amd.build   (or call build()).
Every HIP source is compiled for gfx950 with packed-fp32 instructions disabled;
the host-only table code is compiled by the same driver.  The shared library
lands next to this file, where the binding loads it.
"""
import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(HERE, "libkvk.so")
OBJDIR = os.path.join(ROOT, "_build")
SOURCES = ["table.cpp", "compress.hip", "decode.hip", "mla.hip", "snapkv.hip", "selector.hip",
           "prompt.hip", "keep.hip", "chunk.hip", "rotary.hip", "index.hip", "blocks.hip", "copy.hip"]

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wno-unused-result", "-I", INCLUDE, "-I", CSRC,
]


# Per-source flags.  The selector's attention kernel rescales its product
# accumulators on the VALU now and then; with the accumulators in AGPRs the compiler
# copies them to VGPRs and back on every loop iteration, so its MFMAs write VGPRs; the
# prompt, chunk and block kernels do the same, and the index kernel's minima run over what its MFMAs write.
EXTRA = {src: ["-mllvm", "-amdgpu-mfma-vgpr-form"] for src in ("selector.hip", "prompt.hip", "chunk.hip", "blocks.hip", "index.hip")}


def _compile(src: str) -> str:
    obj = os.path.join(OBJDIR, os.path.basename(src) + ".o")
    lang = ["-x", "hip"] if src.endswith(".hip") else []
    cmd = [HIPCC, *FLAGS, *EXTRA.get(src, []), *lang, "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed on {src}:\n{r.stderr}")
    return obj


def build(verbose: bool = False) -> str:
    os.makedirs(OBJDIR, exist_ok=True)
    with ThreadPoolExecutor(max_workers=min(8, len(SOURCES))) as ex:
        objs = list(ex.map(_compile, SOURCES))
    tmp = LIB + ".tmp"
    cmd = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", *objs, "-o", tmp]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stderr}")
    os.replace(tmp, LIB)
    if verbose:
        print(f"built {LIB}")
    return LIB


if __name__ == "__main__":
    build(verbose=True)
    sys.exit(0)
