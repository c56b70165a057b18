"""Compile the HIP library (csrc/*.hip) for gfx950 into libspike_proj.so,
in-tree next to this file.  Run ``python -m paper_2606_03026_amd.build``."""
from __future__ import annotations

import glob
import os
import subprocess
import sys
import tempfile
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
LIB = os.path.join(HERE, "libspike_proj.so")
SOURCES = [os.path.join(HERE, "csrc", f) for f in (
    "spike_proj.hip", "dense_proj.hip", "quantize.hip", "head_verify.hip",
    "dense_fused.hip", "spike_embed.hip", "head_draft.hip", "head_logits.hip", "spike_clip.hip")]
DEPS = sorted(glob.glob(os.path.join(HERE, "csrc", "*"))) + sorted(glob.glob(os.path.join(ROOT, "include", "*.h")))

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = [
    "--offload-arch=gfx950",
    "-O3",
    "-std=c++17",
    "-fPIC",
    "-shared",
    # no packed FP32 instructions; no contraction or flushing in the
    # FP32 epilogue, which must be one IEEE multiply
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-ffp-contract=off",
    "-fno-gpu-flush-denormals-to-zero",
    "-Wall",
    "-I", os.path.join(ROOT, "include"),
]


def _run(cmd) -> str:
    """Runs a compiler command; its messages."""
    res = subprocess.run(cmd, capture_output=True, text=True)
    # The target feature is a device-pass option: the host (x86) pass of the
    # same hipcc line does not know it and says so once per source.  The
    # device code is built without packed FP32 instructions.
    noise = "'-packed-fp32-ops' is not a recognized feature"
    msgs = "\n".join(l for l in (res.stdout + res.stderr).splitlines() if noise not in l)
    if res.returncode != 0:
        raise RuntimeError(f"hipcc failed ({res.returncode}):\n{' '.join(cmd)}\n{msgs}")
    return msgs


def build(verbose: bool = False) -> str:
    """Sources to objects side by side (one of them takes most of the time), then the library."""
    compile_flags = [f for f in FLAGS if f != "-shared"]
    with tempfile.TemporaryDirectory(prefix="spike_proj_") as tmp:
        objects = [os.path.join(tmp, os.path.basename(s) + ".o") for s in SOURCES]
        with ThreadPoolExecutor(max_workers=min(8, len(SOURCES))) as ex:
            msgs = list(ex.map(lambda so: _run([HIPCC, *compile_flags, "-c", so[0], "-o", so[1]]), zip(SOURCES, objects)))
        lib = LIB + f".tmp{os.getpid()}"
        msgs.append(_run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", *objects, "-o", lib]))
    if verbose and any(m.strip() for m in msgs):
        print("\n".join(m for m in msgs if m.strip()), file=sys.stderr)
    os.replace(lib, LIB)
    return LIB


def is_stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    return any(os.path.getmtime(p) > t for p in DEPS)


if __name__ == "__main__":
    print(build(verbose=True))
