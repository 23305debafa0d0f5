"""AddressSanitizer + UndefinedBehaviorSanitizer build of the entry points over rows of logits (CPU only).

`rp_logits.hip`, checks and launches, is linked with `tests/native/sanitize_rows.cpp`, which stands in for the launches,
and run. The sanitizer flags apply to the host pass only. Any sanitizer report or failed expectation fails the test.
"""
import os

import pytest

from paper_2606_26997_amd import build as B
from tests.test_sanitize_host import CLANG, HOST_SAN, _run

DRIVER = os.path.join(os.path.dirname(os.path.abspath(__file__)), "native", "sanitize_rows.cpp")


def test_rows_of_logits_under_asan_and_ubsan(tmp_path):
    if not os.path.exists(CLANG):
        pytest.skip("ROCm clang++ not found")
    flags = [f for f in B.HIPCC_FLAGS if f != "-O3"] + ["-O1", "-g"]
    objs = []
    for src in (os.path.join(B.CSRC, "rp_logits.hip"), DRIVER):
        objs.append(str(tmp_path / (os.path.basename(src) + ".o")))
        rc, log = _run([B.hipcc(), *flags, *HOST_SAN, "-x", "hip", "-c", src, "-o", objs[-1]])
        assert rc == 0, log
    exe = str(tmp_path / "sanitize_rows")
    rc, log = _run([B.hipcc(), f"--offload-arch={B.ARCH}", "-fsanitize=address", "-fsanitize=undefined",
                    "-fno-gpu-sanitize", *objs, "-o", exe])
    assert rc == 0, log
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0:halt_on_error=1",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    rc, log = _run([exe], env=env, timeout=120)
    assert rc == 0, log
    assert "all expectations held" in log and "runtime error" not in log and "AddressSanitizer" not in log, log
