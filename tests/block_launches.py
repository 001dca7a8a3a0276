"""What the gated projections' gradients launch, on a machine without a GPU (tests/launches_block.cpp)."""

import hashlib
import os
import subprocess
import tempfile

from paper_2505_04846_amd import build as B

SOURCE = os.path.join(os.path.dirname(os.path.abspath(__file__)), "launches_block.cpp")


def _recorder():
    lib = os.path.join(B.PKG_DIR, B.LIB_NAME)
    h = hashlib.sha256()
    for path in (SOURCE, os.path.join(B.CSRC, "kernels.h"), os.path.join(B.INCLUDE, "hiperrag.h")):
        with open(path, "rb") as f:
            h.update(f.read())
    out = os.path.join(B.BUILD_DIR, "launches")
    exe = os.path.join(out, "block_" + h.hexdigest()[:16])
    if os.path.exists(exe):
        return exe
    os.makedirs(out, exist_ok=True)
    with tempfile.TemporaryDirectory(dir=out) as tmp:
        made = os.path.join(tmp, "exe")
        rocm = os.path.dirname(os.path.dirname(B._hipcc()))
        for cmd in ([B._hipcc(), *B.COMMON_FLAGS, "-c", SOURCE, "-o", made + ".o"],
                    ["g++", made + ".o", lib, "-rdynamic", "-o", made, f"-L{rocm}/lib", "-lamdhip64",
                     f"-Wl,-rpath,{rocm}/lib", "-Wl,-rpath," + B.PKG_DIR]):
            r = subprocess.run(cmd, capture_output=True, text=True)
            if r.returncode:
                raise RuntimeError(f"{cmd[0]} failed:\n{r.stderr[-3000:]}")
        os.replace(made, exe)
    return exe


def gradients(n, k, f, dtype=0, packed=False, dx=True, dw=True):
    """[(kernel, workgroups, threads, offset of the columns' maxima or None), ...] of gated_linear_bwd; dtype 0 bf16,
    1 fp16."""
    args = [n, k, f, dtype, int(packed), int(dx) + 2 * int(dw)]
    r = subprocess.run([_recorder(), *map(str, args)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stderr[-2000:]
    *lines, status = r.stdout.splitlines()
    assert status == "status HPR_OK", r.stdout
    return [(w[0], int(w[1]), int(w[2]), int(w[3]) if len(w) > 3 else None) for w in map(str.split, lines)]
