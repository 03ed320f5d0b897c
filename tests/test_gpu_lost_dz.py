"""Behind a wait that ran out dz is NaN in every word, not in some: dw of a word is a sum of that word's entries only.  Built with
nvcc around the kernels' own step; nothing waits here."""
import os
import subprocess

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_every_word_of_a_lost_tile_is_nan(tmp_path):
    nvcc, exe = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc"), str(tmp_path / "lost")
    subprocess.run([nvcc, "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-o", exe, os.path.join(ROOT, "tests", "lost_dz.cu")],
                   check=True)
    lines = subprocess.run([exe], check=True, capture_output=True, text=True, timeout=60).stdout.split("\n")
    # 32 rows or 16, 32 words or 20
    for i, line in enumerate(lines[:8]):
        inside = (16 if i & 2 else 32) * (20 if i & 4 else 32)
        want = [0, 1024 - inside, inside, 0]
        assert list(map(int, line.split())) == ([inside, 1024 - inside, 0, 0] if i & 1 else want)
