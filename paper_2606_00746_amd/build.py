"""Build libgspn.so in place with hipcc for gfx950."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libgspn.so")
SOURCES = ["api.cpp", "scan_tiny.hip", "scan_small.hip", "scan_med_64.hip", "scan_med_56.hip",
           "scan_med_48.hip", "scan_med_40_32_24.hip", "scan_med.hip", "scan_pm.hip",
           "scan_wide.hip", "scan_norm.hip", "scan_plane.hip", "scan_line.hip", "scan_general.hip", "latent.hip",
           "mixers_api.cpp", "qk_norm.hip", "attn_fwd.hip", "attn_bwd.hip", "attn_bwd_f32.hip", "attn_split.hip",
           "delta_fwd.hip", "delta_bwd.hip", "delta_bf16.hip"]
ARCH = "gfx950"

HIPCC_FLAGS = [
    f"--offload-arch={ARCH}", "-O3", "-fPIC", "-std=c++17", "-Wall",
    # never let the compiler form packed fp32 ops (v_pk_*_f32)
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-I", os.path.join(HERE, "..", "include"),
]

# Attention's bf16 gradient kernels keep up to 128 accumulator registers a lane beside as
# many operands: with results of matrix instructions in vector registers the compiler
# does not copy them between the two register files around every tile (key gradients
# at heads of 128: 628 -> 398 us).
SOURCE_FLAGS = {"attn_bwd.hip": ["-mllvm", "-amdgpu-mfma-vgpr-form=true"]}


def hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found")


def build(verbose: bool = False, jobs: int = 0, incremental: bool = False) -> str:
    """Compiles every source (incremental: only those older than their object,
    counting the shared headers) and links libgspn.so in place."""
    cc = hipcc()
    if jobs <= 0:
        jobs = max(1, min(8, os.cpu_count() or 1))
    objdir = os.path.join(HERE, "_build")
    os.makedirs(objdir, exist_ok=True)

    headers = [os.path.join(CSRC, h) for h in os.listdir(CSRC) if h.endswith((".hpp", ".h"))]
    headers.append(os.path.join(HERE, "..", "include", "gspn.h"))
    newest_header = max(os.path.getmtime(h) for h in headers)

    def compile_one(src):
        obj = os.path.join(objdir, os.path.splitext(src)[0] + ".o")
        if incremental and os.path.exists(obj):
            t = os.path.getmtime(obj)
            if t > os.path.getmtime(os.path.join(CSRC, src)) and t > newest_header:
                return obj
        lang = ["-x", "hip"]
        cmd = [cc, *HIPCC_FLAGS, *SOURCE_FLAGS.get(src, []), *lang, "-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        r = subprocess.run(cmd, capture_output=True, text=True)
        msgs = [ln for ln in (r.stderr or "").splitlines()
                if "packed-fp32-ops" not in ln and ln.strip()]
        if r.returncode != 0:
            raise RuntimeError(f"hipcc failed on {src}:\n" + "\n".join(msgs))
        if verbose and msgs:
            print("\n".join(msgs))
        return obj

    with ThreadPoolExecutor(max_workers=jobs) as ex:
        objs = list(ex.map(compile_one, SOURCES))
    tmp = LIB + ".tmp"
    cmd = [cc, f"--offload-arch={ARCH}", "-shared", "-fPIC", "-o", tmp, *objs]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)
    os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv, jobs=8, incremental="-i" in sys.argv))
