"""Builds libinfmllm.so (the C-ABI library of hand-written gfx950 kernels) in-tree with hipcc.

    python -m paper_2409_09086_amd.build

hipcc cross-compiles for gfx950 without a GPU.  The shared library lands next to this file
so that it travels with the source tree; nothing is installed.
"""
import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libinfmllm.so")
SOURCES = ["api.hip", "cache_kernels.hip", "attn_simple.hip", "attn_f32.hip", "attn_mfma.hip", "attn_mfma64.hip", "attn_rows.hip", "attn_rows64.hip", "decode_attn.hip", "rope.hip", "select_kernel.hip",
           "rotary.hip", "paged_rows.hip", "paged_fwd.hip", "paged_mixed.hip", "paged_api.hip"]
# packed-fp32 instructions are switched off for every device pass
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Wall",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]


def _compile(src, verbose):
    obj = os.path.join(OBJ, src.replace(".hip", ".o"))
    cmd = ["hipcc", *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    err = "\n".join(l for l in r.stderr.splitlines() if "packed-fp32-ops" not in l or "error" in l)
    if r.returncode != 0:
        raise RuntimeError("hipcc failed on %s:\n%s" % (src, r.stderr))
    if verbose and err.strip():
        print(err, file=sys.stderr)
    return obj


def build(verbose=True):
    os.makedirs(OBJ, exist_ok=True)
    with ThreadPoolExecutor(max_workers=min(8, len(SOURCES))) as ex:
        objs = list(ex.map(lambda s: _compile(s, verbose), SOURCES))
    tmp = LIB + ".tmp.%d" % os.getpid()
    subprocess.check_call(["hipcc", "--offload-arch=gfx950", "-shared", "-fPIC", "-o", tmp, *objs])
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build())
