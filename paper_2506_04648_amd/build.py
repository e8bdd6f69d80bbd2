"""Builds libfps.so (the C-ABI library) in-tree with hipcc for gfx950."""
from __future__ import annotations

import os
import subprocess
import tempfile
from concurrent.futures import ThreadPoolExecutor

_HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(_HERE)
CSRC = os.path.join(_HERE, "csrc")
SOURCES = ("fps_host.cpp", "fps_layout.hip", "fps_quantize.hip", "fps_attn.hip",
           "fps_attn_fp8.hip", "fps_attn_bf16.hip", "fps_issue_mix.hip", "fps_host_operators.cpp", "fps_rotate.hip",
           "fps_mx4.hip", "fps_mx4_matmul.hip")
# accumulators in AGPRs: a wave's 256 are as many as there are architectural registers, and no vector code reads them before the end
AGPR_SOURCES = ("fps_mx4_matmul.hip",)
OUT = os.path.join(_HERE, "libfps.so")


def build_lib(verbose: bool = False) -> str:
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    flags = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-I" + os.path.join(ROOT, "include"),
             # packed fp32 instructions stay off (they are generated from ordinary float code otherwise)
             "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
             # no NaN ever enters the attention (inputs are finite, masked scores are -inf, never inf-inf): lets fmax/fmin
             # compile without the canonicalising v_max(x,x) in front of every operand; what
             # may meet one, around the attention and on the host, compares bits
             "-fno-honor-nans"] + os.environ.get("FPS_EXTRA_HIPCC_FLAGS", "").split()
    # MFMA results stay in architectural VGPRs: the softmax VALU code reads them directly instead of through
    # v_accvgpr moves
    vgpr_form = ["-mllvm", "-amdgpu-mfma-vgpr-form"]

    def run(cmd):
        res = subprocess.run(cmd, capture_output=True, text=True)
        if verbose or res.returncode != 0:
            print(res.stdout)
            print("\n".join(l for l in res.stderr.splitlines() if "packed-fp32-ops" not in l))
        if res.returncode != 0:
            raise RuntimeError("hipcc failed building libfps.so")

    # each source to an object of its own, which the link takes alone: behind a source hipcc takes an object for one as well
    with tempfile.TemporaryDirectory() as tmp, ThreadPoolExecutor(8) as pool:
        objects = [os.path.join(tmp, s + ".o") for s in SOURCES]
        jobs = [pool.submit(run, [hipcc, *flags, *([] if s in AGPR_SOURCES else vgpr_form), "-c", os.path.join(CSRC, s), "-o", o])
                for s, o in zip(SOURCES, objects)]
        for job in jobs:
            job.result()
        run([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", OUT] + objects)
    return OUT
