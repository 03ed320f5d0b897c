"""A kernel's limit of dynamic shared memory, set by several threads at once.  Built with nvcc, run on the host."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_limit_holds_whoever_sets_it_last(tmp_path):
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    exe = str(tmp_path / "race")
    subprocess.run([nvcc, "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-o", exe,
                    os.path.join(ROOT, "tests", "smem_limit_race.cu")], check=True)
    lines = subprocess.run([exe], check=True, capture_output=True, text=True, timeout=60).stdout.split("\n")
    ok, attribute, wanted = map(int, lines[0].split())
    assert ok and attribute >= wanted
    assert lines[1] == "0", "more than a block may have was not refused"
