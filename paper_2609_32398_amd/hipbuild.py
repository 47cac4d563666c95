"""Build libdoloss.so (HIP, gfx950) in-tree with hipcc."""
from __future__ import annotations

import os
import subprocess
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB_PATH = os.path.join(HERE, "libdoloss.so")
SOURCES = ["api.hip", "topk.hip", "topk_ragged.hip", "topk_pieces.hip", "topk_wide.hip", "reduce.hip", "surrogate.hip", "loadstats.hip", "rem.hip",
           "expert_api.hip", "expert_rows.hip", "expert_matmul_bf16.hip", "expert_matmul_f32.hip", "expert_wgrad_bf16.hip", "expert_wgrad_f32.hip", "expert_swiglu.hip", "expert_skinny.hip", "act8.hip",
           "fp8.hip", "expert_matmul_fp8.hip", "expert_swiglu_fp8.hip", "expert_layer.hip"]

HIPCC_FLAGS = [
    "--offload-arch=gfx950",
    "-O3",
    "-std=c++17",
    "-fPIC",
    "-fvisibility=hidden",
    # keep the compiler from forming packed-FP32 instructions
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
]


def _run(cmd) -> str:
    res = subprocess.run(cmd, capture_output=True, text=True)
    out = "\n".join(l for l in (res.stdout + res.stderr).splitlines() if "packed-fp32-ops" not in l)
    if res.returncode != 0:
        raise RuntimeError(f"hipcc failed ({res.returncode}):\n{out}")
    return out.strip()


def build(verbose: bool = False) -> str:
    """Compile every HIP source of the library; returns the path of the .so."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    tmp = LIB_PATH + ".tmp"
    with tempfile.TemporaryDirectory() as d:
        objs = [os.path.join(d, s + ".o") for s in SOURCES]
        cmds = [[hipcc, *HIPCC_FLAGS, "-c", os.path.join(CSRC, s), "-o", o] for s, o in zip(SOURCES, objs)]
        with ThreadPoolExecutor(min(len(cmds), os.cpu_count() or 1)) as pool:
            out = list(pool.map(_run, cmds))
        out.append(_run([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", *objs, "-o", tmp]))
    if verbose and any(out):
        print("\n".join(o for o in out if o))
    os.replace(tmp, LIB_PATH)
    return LIB_PATH


if __name__ == "__main__":
    print(build(verbose=True))
