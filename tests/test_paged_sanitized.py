"""The host side of the paged cache's entry points built with AddressSanitizer and UndefinedBehaviorSanitizer on the host
code and driven by a small native program: 300 000 random pools and parameter sets.  Nothing is launched."""
import os
import subprocess

import pytest

from paper_2502_17599_amd.build import HIPCC_FLAGS, PKG_DIR, ROOT

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not available")
def test_paged_validation_under_sanitizers(tmp_path):
    exe = tmp_path / "paged_sanitizer_check"
    flags = [f for f in HIPCC_FLAGS if f not in ("-O3", "-fPIC")]
    cmd = [HIPCC, *flags, "-O1", "-g", "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-sanitize-recover=undefined", "-I", os.path.join(ROOT, "include"),
           os.path.join(ROOT, "tests", "native", "paged_sanitizer_check.cpp"),
           *(os.path.join(PKG_DIR, "csrc", f + ".hip") for f in ("page_tables", "rotary_kernels", "paged_store", "paged_attention")),
           "-o", str(exe)]
    build = subprocess.run(cmd, capture_output=True, text=True)
    assert build.returncode == 0, build.stderr[-3000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    run = subprocess.run([str(exe)], capture_output=True, text=True, env=env, timeout=300)
    assert run.returncode == 0, (run.stdout + run.stderr)[-3000:]
    assert "paged sanitizer check ok" in run.stdout
    assert "runtime error" not in run.stderr and "AddressSanitizer" not in run.stderr
