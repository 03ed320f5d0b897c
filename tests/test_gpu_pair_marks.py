"""A wait that runs out in one of two blocks that form a tile together: either's results are built from both blocks' operands, so
both have to know.  Built with nvcc; the wait has few tries and ends by itself."""
import os
import subprocess

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_a_wait_that_runs_out_marks_both_blocks(tmp_path):
    nvcc, exe = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc"), str(tmp_path / "marks")
    subprocess.run([nvcc, "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-o", exe, os.path.join(ROOT, "tests", "pair_marks.cu")],
                   check=True)
    lines = subprocess.run([exe], check=True, capture_output=True, text=True, timeout=60).stdout.split("\n")
    assert lines[:3] == ["1 1 4", "1 1 4", "0 0 0"]
