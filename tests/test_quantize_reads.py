"""The quantiser's wide loads stay inside the matrix, on the CPU: the kernel's own conditions (csrc/fp8.h) over every small
number of rows, columns and every row stride; tests/host_sanitize/quant_reads.cpp counts."""
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")
def test_no_piece_ends_behind_the_last_row(tmp_path):
    exe = str(tmp_path / "quant_reads")
    subprocess.run(["hipcc", "--offload-arch=gfx950", "--cuda-host-only", "-O1", "-std=c++17", "-x", "hip",
                    os.path.join(HERE, "host_sanitize", "quant_reads.cpp"), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout
