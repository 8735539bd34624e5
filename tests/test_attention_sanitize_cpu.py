"""The attention calls' boundary (csrc/attention_api.cpp: validation, sizes, overlaps) under AddressSanitizer and
UndefinedBehaviorSanitizer, host code only: built with tests/sanitize/attention_driver.cpp, whose stand-ins take the
place of the launches."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2506_13771_amd", "csrc")
HIPCC = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
SAN = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined"]


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc missing")
def test_attention_boundary_under_sanitizers(tmp_path):
    flags = ["-x", "hip", "--offload-host-only", "-O1", "-g", "-std=c++17", "-fno-omit-frame-pointer", "-I", os.path.join(ROOT, "include")]
    objs = []
    for src in (os.path.join(CSRC, "attention_api.cpp"), os.path.join(ROOT, "tests", "sanitize", "attention_driver.cpp")):
        objs.append(str(tmp_path / (os.path.basename(src) + ".o")))
        subprocess.run([HIPCC] + flags + SAN + ["-c", src, "-o", objs[-1]], check=True)
    exe = str(tmp_path / "driver")
    subprocess.run([HIPCC] + SAN + ["--offload-arch=gfx950"] + objs + ["-o", exe], check=True)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    res = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=120)
    assert res.returncode == 0 and "sanitized attention checks passed" in res.stdout, res.stdout + res.stderr
    assert "runtime error" not in res.stderr and "AddressSanitizer" not in res.stderr, res.stderr
