"""CPU test of the rules that products of rows are launched by (csrc/sc_rules.h): tests/native/product_rules.cpp compiles, with its assertions, and runs."""
import os
import subprocess

from paper_2402_07710_amd import build


def test_rules_of_products(tmp_path):
    source, program = os.path.join(os.path.dirname(os.path.abspath(__file__)), "native", "product_rules.cpp"), str(tmp_path / "product_rules")
    made = subprocess.run([build.CXX, "-std=c++17", "-O1", "-Wall", "-Werror", "-I", build.CSRC, source, "-o", program], capture_output=True, text=True)
    assert made.returncode == 0, made.stderr[-3000:]
    run = subprocess.run([program], capture_output=True, text=True, timeout=60)
    assert run.returncode == 0, run.stdout
