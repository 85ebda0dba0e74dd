"""CPU test of the rules that attention and the group norm are launched by (csrc/sc_rules.h): tests/native/attention_rules.cpp compiles, with its assertions, and runs."""
import os
import subprocess

from paper_2402_07710_amd import build


def test_rules_of_attention_and_norm(tmp_path):
    source, program = os.path.join(os.path.dirname(os.path.abspath(__file__)), "native", "attention_rules.cpp"), str(tmp_path / "attention_rules")
    made = subprocess.run([build.CXX, "-std=c++17", "-O1", "-Wall", "-Werror", "-I", build.CSRC, source, "-o", program], capture_output=True, text=True)
    assert made.returncode == 0, made.stderr[-3000:]
    run = subprocess.run([program], capture_output=True, text=True, timeout=60)
    assert run.returncode == 0, run.stdout


def test_operands_that_meet(tmp_path):
    source, program = os.path.join(os.path.dirname(os.path.abspath(__file__)), "native", "heads.cpp"), str(tmp_path / "heads")
    include = os.path.join(build.ROOT, "include")
    made = subprocess.run([build.CXX, "-std=c++17", "-O1", "-Wall", "-Werror", "-I", build.CSRC, "-I", include, source, "-o", program], capture_output=True, text=True)
    assert made.returncode == 0, made.stderr[-3000:]
    run = subprocess.run([program], capture_output=True, text=True, timeout=60)
    assert run.returncode == 0, run.stdout
