"""Single calls around the latent cache against stand-ins of the launchers (no GPU): what reaches a launch, and what does not."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not found")
    csrc, exe = os.path.join(ROOT, "paper_2609_37626_amd", "csrc"), tmp_path_factory.mktemp("layer") / "layer_calls"
    r = subprocess.run([hipcc, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17",
                        "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
                        "-Xarch_host", "-fno-sanitize-recover=undefined", "-I", os.path.join(ROOT, "include"), "-I", csrc,
                        os.path.join(csrc, "api.cpp"), os.path.join(csrc, "layer_api.cpp"),
                        os.path.join(ROOT, "tests", "sanitize", "launch_stubs.cpp"),
                        os.path.join(ROOT, "tests", "sanitize", "layer_calls.cpp"), "-o", str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]

    def run(what):
        env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=1", UBSAN_OPTIONS="print_stacktrace=1")
        r = subprocess.run([str(exe), what], capture_output=True, text=True, env=env, timeout=300)
        assert r.returncode == 0 and r.stdout.startswith("ok "), r.stdout + r.stderr[-4000:]
        return int(r.stdout.split()[1])

    return run


def test_a_stride_over_a_dimension_of_one_is_not_looked_at(driver):
    assert driver("strides") > 60
