"""Where the stretches of prompt attention run, computed on the host by the function that the kernels use (prompt_map_host.cpp)."""
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="no hipcc")
def test_the_stretches_in_use_lie_on_all_xcds(tmp_path):
    exe = str(tmp_path / "prompt_map_host")
    subprocess.run([HIPCC, "-x", "hip", "--offload-host-only", "-std=c++17", "-O1", "-o", exe, os.path.join(HERE, "prompt_map_host.cpp")], check=True)
    got = subprocess.run([exe], stdout=subprocess.PIPE, text=True)
    assert got.returncode == 0, got.stdout
