"""CPU test of how weight gradients are cut into parts at the largest sizes (csrc/sc_rules.h): tests/native/weight_parts.cpp compiles and runs."""
import os
import subprocess

from paper_2402_07710_amd import build


def test_parts_of_the_largest_weight_gradients(tmp_path):
    source, program = os.path.join(os.path.dirname(os.path.abspath(__file__)), "native", "weight_parts.cpp"), str(tmp_path / "weight_parts")
    made = subprocess.run([build.CXX, "-std=c++17", "-O1", "-Wall", "-Werror", "-I", build.CSRC, source, "-o", program], capture_output=True, text=True)
    assert made.returncode == 0, made.stderr[-3000:]
    run = subprocess.run([program], capture_output=True, text=True, timeout=60)
    assert run.returncode == 0, run.stdout
