"""Builds libdnb.so (HIP kernels + C ABI) for gfx950 with hipcc, in tree."""
from __future__ import annotations

import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libdnb.so")
SOURCES = ["dnb_elem.hip", "dnb_conv_f32.hip", "dnb_conv_f32_fast.hip", "dnb_conv3x3_f32.hip", "dnb_bwd_f32.hip", "dnb_nhwc_bf16.hip", "dnb_nhwc_conv1.hip", "dnb_nhwc_conv3.hip", "dnb_nhwc_bwd.hip", "dnb_nhwc_wgrad.hip",
           "dnb_block.hip", "dnb_net.hip", "dnb_inet.hip",
           "dnb_attn.hip", "dnb_attn_bwd.hip", "dnb_rope.hip", "dnb_norm.hip", "dnb_clip.hip",
           "dnb_paged_attn.hip", "dnb_qk.hip", "dnb_pages.hip"]
# Packed-fp32 instruction selection is switched off for all device code on this target.
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Wall", "-Wno-unused-function",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]

# Products write their results to the registers that other instructions read: with accumulators in registers of their own the
# attention over pages moved sums there and back where paths meet (single tokens over long caches 118 -> 74 us).
MORE_FLAGS = {"dnb_paged_attn.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form=1"]}


def build(verbose: bool = False) -> str:
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    def compile_one(src):
        obj = os.path.join(CSRC, src.replace(".hip", ".o"))
        cmd = [hipcc, *FLAGS, *MORE_FLAGS.get(src, []), "-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            sys.stderr.write(r.stdout + r.stderr)
            raise RuntimeError(f"hipcc failed on {src}")
        return obj

    # the translation units are independent: compile them side by side (a few hundred MB each)
    with ThreadPoolExecutor(max_workers=min(len(SOURCES), os.cpu_count() or 1)) as pool:
        objs = list(pool.map(compile_one, SOURCES))
    cmd = [hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", LIB, *objs]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        sys.stderr.write(r.stdout + r.stderr)
        raise RuntimeError("link failed")
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
