"""CPU test of the units by which a bias' gradient is summed (csrc/sc_rules.h): tests/native/bias_units.cpp compiles, with its assertions, and runs."""
import os
import subprocess

from paper_2402_07710_amd import build


def test_units_of_a_bias(tmp_path):
    source, program = os.path.join(os.path.dirname(os.path.abspath(__file__)), "native", "bias_units.cpp"), str(tmp_path / "bias_units")
    made = subprocess.run([build.CXX, "-std=c++17", "-O1", "-Wall", "-Werror", "-I", build.CSRC, source, "-o", program], capture_output=True, text=True)
    assert made.returncode == 0, made.stderr[-3000:]
    run = subprocess.run([program], capture_output=True, text=True, timeout=60)
    assert run.returncode == 0, run.stdout
