"""AddressSanitizer + UndefinedBehaviorSanitizer over the host code of the operators around a block's layers, as test_sanitizers.py runs it over the other entry points (no GPU)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SAN = os.path.join(ROOT, "tests", "sanitize")
ENV = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")


def _run(cmd, **kw):
    r = subprocess.run(cmd, capture_output=True, text=True, **kw)
    assert r.returncode == 0, f"{' '.join(cmd[:3])} ... failed ({r.returncode}):\n{r.stdout[-3000:]}\n{r.stderr[-6000:]}"
    return r


def test_block_operators_under_address_and_ub_sanitizers(tmp_path):
    from paper_2509_21302_amd import build as B
    if not shutil.which(B.HIPCC) and not os.path.exists(B.HIPCC):
        pytest.skip("hipcc is not installed")
    others = [os.path.join(B.BUILD, os.path.splitext(s)[0] + ".o") for s in B.SOURCES if s != "api.hip"]
    newest = max(os.path.getmtime(os.path.join(B.CSRC, f)) for f in os.listdir(B.CSRC))
    if not all(os.path.exists(o) and os.path.getmtime(o) >= newest for o in others):
        B.build()                               # the other objects carry the kernels that api.hip launches; plain builds of them do
    api, driver, exe = (str(tmp_path / n) for n in ("api.o", "driver.o", "driver"))
    flags = [f for f in B.FLAGS if f != "-O3"]
    _run([B.HIPCC, *flags, "-O1", "-g", "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-c", os.path.join(B.CSRC, "api.hip"), "-o", api])
    _run([B.HIPCC, "-x", "c", "-std=c11", "-O1", "-g", "-I", B.INCLUDE, "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-c", os.path.join(SAN, "block_driver.c"), "-o", driver])
    _run([B.HIPCC, "--offload-arch=gfx950", "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-o", exe, driver, api, *others])
    assert "0 mismatches" in _run([exe], env=ENV).stdout
