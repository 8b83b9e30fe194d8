"""What the kernels' own listings have to show (the compiler runs here, the kernels do not)."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2609_37626_amd import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def listing(source, to):
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not found")
    r = subprocess.run([hipcc] + build.HIPCC_FLAGS + build.SOURCE_FLAGS.get(source, [])
                       + ["--cuda-device-only", "-S", os.path.join(build.CSRC, source), "-o", str(to)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    return to.read_text()


@pytest.mark.parametrize("source", ["mla_prefill.hip", "mla_project.hip"])
def test_the_loads_to_lds_are_alone_with_m0(source, tmp_path):
    """The loads' asm writes M0 and leaves it: each mention of it is theirs, right before a load that takes it."""
    lines = [line.strip() for line in listing(source, tmp_path / "listing").splitlines()]
    mentions = [i for i, line in enumerate(lines) if re.search(r"\bm0\b", line.split(";")[0])]
    assert len(mentions) > 20
    for i in mentions:
        assert re.match(r"s_(sub_u32|mov_b32) m0, ", lines[i]), lines[i]
        assert lines[i + 1] == "s_nop 0" and lines[i + 2].startswith("global_load_lds_dwordx4 "), lines[i:i + 3]
