"""Builds libhiperrag.so (HIP for gfx950) in the package directory.

    python -m paper_2505_04846_amd.build        # or paper_2505_04846_amd.build.build()

Every HIP source is compiled with hipcc for gfx950 only, with packed-fp32 VALU instructions
disabled, and linked into one shared library with a plain C ABI (include/hiperrag.h).
"""

import concurrent.futures
import os
import shutil
import subprocess
import sys

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG_DIR)
CSRC = os.path.join(PKG_DIR, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD_DIR = os.path.join(PKG_DIR, "_build")
LIB_NAME = "libhiperrag.so"
ARCH = "gfx950"

SOURCES = ["abi.hip", "maxsim.hip", "maxsim_argmax.hip", "topk.hip", "loss.hip", "contrastive.hip",
           "dense.hip", "chunking.hip", "calibration.hip", "attention.hip", "adapters.hip", "rotary.hip"]


def _hipcc():
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found (set HIPCC or install ROCm under /opt/rocm)")


COMMON_FLAGS = [
    f"--offload-arch={ARCH}",
    "-O3",
    "-std=c++17",
    "-fPIC",
    "-Wall",
    "-Wno-unused-parameter",
    # keep the compiler from emitting packed fp32 VALU ops (v_pk_{add,mul,fma}_f32)
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    f"-I{INCLUDE}",
    f"-I{CSRC}",
]


# Per-file extra flags.  The MaxSim kernels take inputs that are finite by contract, and the attention kernels q,
# dout and every key row that some query sees (the header states both), so NaN semantics need not be honoured
# there: without this every fmaxf of the running max is preceded by two NaN-quieting self-maxes, tripling the VALU
# work per tile.  Key rows that no query sees may hold NaN.  The attention kernels do not load them, but for the
# 32 keys of a wave of the dk/dv kernel, whose scores and products are replaced by selects before anything is
# computed from them: the flag lets the compiler assume about a value that is used, not about one that a select drops.
FILE_FLAGS = {"maxsim.hip": ["-fno-honor-nans"], "maxsim_argmax.hip": ["-fno-honor-nans"],
              "attention.hip": ["-fno-honor-nans"]}


def _compile(src, verbose):
    obj = os.path.join(BUILD_DIR, os.path.splitext(src)[0] + ".o")
    cmd = [_hipcc(), *COMMON_FLAGS, *FILE_FLAGS.get(src, []), "-c", os.path.join(CSRC, src),
           "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    errs = "\n".join(l for l in (r.stderr or "").splitlines() if "packed-fp32-ops" not in l)
    if r.returncode != 0:
        raise RuntimeError(f"hipcc failed for {src}:\n{errs}")
    if verbose and errs.strip():
        print(errs, file=sys.stderr)
    return obj


def build(verbose=False):
    """Compiles every source and links PKG_DIR/libhiperrag.so.  Always rebuilds."""
    os.makedirs(BUILD_DIR, exist_ok=True)
    srcs = [s for s in SOURCES if os.path.exists(os.path.join(CSRC, s))]
    with concurrent.futures.ThreadPoolExecutor(max_workers=min(8, len(srcs))) as ex:
        objs = list(ex.map(lambda s: _compile(s, verbose), srcs))
    out = os.path.join(PKG_DIR, LIB_NAME)
    tmp = out + ".tmp"
    cmd = [_hipcc(), f"--offload-arch={ARCH}", "-shared", "-fPIC", *objs, "-o", tmp]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stderr}")
    os.replace(tmp, out)
    return out


if __name__ == "__main__":
    print(build(verbose=True))
