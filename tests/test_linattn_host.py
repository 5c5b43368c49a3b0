"""The launches that the linear-attention entry points make, looked at without a GPU (tests/linattn_host_driver.cpp)."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.timeout(300)
def test_launches(tmp_path):
    exe = str(tmp_path / "driver")
    cmd = [os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), "-x", "hip", "--offload-arch=gfx950", "--offload-host-only", "-std=c++17", "-O1",
           "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fsanitize-trap=undefined", os.path.join(ROOT, "tests", "linattn_host_driver.cpp"),
           "-o", exe, "-Wl,--unresolved-symbols=ignore-all"]          # (the device code it has none of)
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and "0 failures" in r.stdout, r.stdout[-3000:]
