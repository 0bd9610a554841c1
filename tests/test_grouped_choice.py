"""Which kernel zipmoe_grouped_matmul takes is decided by plain C++ on sizes; this compiles it with g++ and holds it to
measured times of both kernels."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_kernel_taken_is_not_the_slower_one(tmp_path):
    exe = str(tmp_path / "grouped_choice_check")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-I", os.path.join(ROOT, "paper_2601_21198_b200", "csrc"),
                           os.path.join(ROOT, "tests", "csrc", "grouped_choice_check.cpp"), "-o", exe])
    out = subprocess.run([exe], capture_output=True, text=True)
    assert out.returncode == 0 and out.stdout.strip() == "ok", out.stdout
