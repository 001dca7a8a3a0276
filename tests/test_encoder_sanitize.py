"""CPU-only: the encoder operators' host code (argument checks, size queries, the rules that choose
kernels, workspace carving) under AddressSanitizer and UndefinedBehaviorSanitizer, driven by
tests/abi_sanitize_encoder.cpp against the objects that test_abi_sanitize builds."""

import hashlib
import os
import shutil
import subprocess

import pytest

from paper_2505_04846_amd import build as B
from test_abi_sanitize import HERE, OUT, SAN, _build

DRIVER = os.path.join(HERE, "abi_sanitize_encoder.cpp")


def _driver():
    library = os.path.dirname(_build())
    with open(DRIVER, "rb") as f:
        exe = os.path.join(library, "encoder_" + hashlib.sha256(f.read()).hexdigest()[:16])
    if os.path.exists(exe):
        return exe
    hipcc = B._hipcc()
    obj = exe + ".driver"
    objs = [os.path.join(OUT, os.path.splitext(s)[0] + ".o") for s in B.SOURCES]
    rocm = os.path.dirname(os.path.dirname(hipcc))
    for cmd in ([hipcc, *B.COMMON_FLAGS, *SAN, "-c", DRIVER, "-o", obj],
                ["g++", *objs, obj, "-fsanitize=address,undefined", "-o", exe, f"-L{rocm}/lib",
                 f"-Wl,-rpath,{rocm}/lib", "-lamdhip64"]):
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode:
            raise RuntimeError(f"{cmd[0]} failed:\n{r.stderr[-3000:]}")
    return exe


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++ for the host link")
@pytest.mark.skipif(os.path.exists("/dev/kfd"), reason="for machines without a GPU: the driver "
                    "calls entry points with fake device pointers")
def test_encoder_host_code_under_asan_and_ubsan():
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    r = subprocess.run([_driver()], capture_output=True, text=True, env=env, timeout=300)
    assert r.returncode == 0, f"{r.stdout}\n{r.stderr[-4000:]}"
    assert "ok: 0 failures" in r.stdout
