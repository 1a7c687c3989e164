"""The workspace of attention over the 4-bit cache: taken once for the largest batch, it serves every smaller one, as the other operators' do."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


@pytest.mark.skipif(shutil.which(HIPCC) is None, reason="hipcc not found")
def test_a_workspace_serves_smaller_batches(tmp_path):
    exe = str(tmp_path / "driver")
    res = subprocess.run([HIPCC, "-O1", "-std=c++17", "--offload-arch=gfx950", "-Wno-unused-command-line-argument", "-o", exe,
                          os.path.join(ROOT, "paper_2605_25655_amd", "csrc", "kv4_api.hip"), "-x", "hip", os.path.join(ROOT, "tests", "plan", "kv4_workspace_driver.cpp")],
                         capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-4000:]
    res = subprocess.run([exe], capture_output=True, text=True)
    assert res.returncode == 0 and res.stdout.startswith("ok "), (res.returncode, res.stdout)
