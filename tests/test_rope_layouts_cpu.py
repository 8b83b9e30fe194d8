"""splash_rope's layouts of y: rows that overlap are refused, all others taken (no GPU)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_rope_refuses_exactly_the_layouts_whose_rows_overlap(tmp_path):
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not found")
    csrc, exe = os.path.join(ROOT, "paper_2609_37626_amd", "csrc"), tmp_path / "rope_layouts"
    r = subprocess.run([hipcc, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17",
                        "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
                        "-Xarch_host", "-fno-sanitize-recover=undefined", "-I", os.path.join(ROOT, "include"), "-I", csrc,
                        os.path.join(csrc, "api.cpp"), os.path.join(csrc, "step_api.cpp"),
                        os.path.join(ROOT, "tests", "sanitize", "launch_stubs.cpp"),
                        os.path.join(ROOT, "tests", "sanitize", "rope_layouts.cpp"), "-o", str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=1", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([str(exe)], capture_output=True, text=True, env=env, timeout=300)
    assert r.returncode == 0, r.stderr[-4000:]
    ok, accepted, refused = r.stdout.split()
    assert ok == "ok" and int(accepted) > 1000 and int(refused) > 1000
