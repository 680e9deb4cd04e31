"""Index rules of the kernels over a cache of keys, run on the host: tests/host_checks_tiles.cpp over csrc/attention.h."""
import os
import subprocess

from paper_2602_16052_amd import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_no_place_behind_the_last_key_is_read_from_memory(tmp_path):
    exe = str(tmp_path / "host_checks_tiles")
    cc = subprocess.run([build.hipcc_path(), "-x", "hip", "--offload-host-only", "--offload-arch=gfx950", "-std=c++17", "-O1",
                         "-I", os.path.join(ROOT, "include"), "-I", build.CSRC,
                         os.path.join(ROOT, "tests", "host_checks_tiles.cpp"), "-o", exe],
                        stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert cc.returncode == 0, cc.stdout
    run = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=60)
    assert run.returncode == 0, run.stdout
    assert "host checks passed" in run.stdout
