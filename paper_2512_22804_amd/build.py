"""Compile the HIP library for gfx950 (MI355X) in-tree: ``python -m paper_2512_22804_amd.build``.

hipcc cross-compiles without a GPU.  Flags that matter for correctness:
  -ffp-contract=off   y = fl32(x*s) must stay one IEEE multiply (never fused into y - q);
  -packed-fp32-ops    disabled target feature: no v_pk_*_f32 instructions are generated.
"""
from __future__ import annotations

import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libmor.so")
SOURCES = ["mor_kernels.hip", "mor_partitions.hip", "mor_api.hip", "mx_quantize.hip", "mx_product.hip", "mx_experts.hip", "mx_api.hip"]
HEADERS = ["mor_device.h", "mor_launch.h", "mor_stream.h", "mor_sub1x128.h", "mor_team.h", "mx_device.h", "mx_launch.h",
           os.path.join("..", "..", "include", "mor.h"), os.path.join("..", "..", "include", "mor_mx.h")]
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-ffp-contract=off", "-fno-fast-math",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-Wall", "-Wno-unused-command-line-argument"]


def build(force: bool = True, verbose: bool = False) -> str:
    srcs = [os.path.join(CSRC, s) for s in SOURCES]
    deps = srcs + [os.path.join(CSRC, h) for h in HEADERS]
    if not force and os.path.exists(LIB) and all(os.path.getmtime(LIB) >= os.path.getmtime(d) for d in deps):
        return LIB
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    noise = ("packed-fp32-ops", "is not a recognized feature")

    def run(cmd):
        if verbose:
            print(" ".join(cmd))
        res = subprocess.run(cmd, capture_output=True, text=True)
        if res.returncode != 0:
            raise RuntimeError("hipcc failed:\n" + res.stderr)
        err = "\n".join(l for l in res.stderr.splitlines() if not any(n in l for n in noise))
        if verbose and err.strip():
            print(err, file=sys.stderr)

    with tempfile.TemporaryDirectory() as tmp:
        objs = [os.path.join(tmp, os.path.basename(s) + ".o") for s in srcs]
        with ThreadPoolExecutor(min(len(srcs), os.cpu_count() or 1)) as pool:
            list(pool.map(lambda so: run([hipcc, *FLAGS, "-c", "-o", so[1], so[0]]), zip(srcs, objs)))
        run([hipcc, *FLAGS, "-shared", "-o", LIB, *objs])
    return LIB


if __name__ == "__main__":
    print(build(force=True, verbose=True))
