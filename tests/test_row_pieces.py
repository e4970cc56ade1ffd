"""Rows of logits as 16-byte pieces, compiled for the host with an address sanitizer: nothing outside the row's elements is
read, and every piece holds what it should (CPU)."""
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)


def test_only_the_rows_elements_are_read(tmp_path):
    nvcc = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(nvcc):
        pytest.skip("nvcc not available")
    exe = str(tmp_path / "row_pieces_host")
    r = subprocess.run([nvcc, "-std=c++17", "-Xcompiler", "-fsanitize=address", "-I", os.path.join(ROOT, "include"), "-I",
                        os.path.join(ROOT, "paper_2607_08406_gb300", "csrc"), "-o", exe,
                        os.path.join(HERE, "row_pieces_host.cu")], capture_output=True, text=True)
    if r.returncode and "asan" in r.stderr:
        pytest.skip("no address sanitizer")
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[:2000]
    assert int(r.stdout) > 10000
