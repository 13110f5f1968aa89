"""The numbers that a speculative step's operators are held in, on the host."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("g++") is None, reason="no C++ compiler")
def test_probabilities_in_fixed_point(tmp_path):
    exe = tmp_path / "tree_fixed"
    cc = subprocess.run(["g++", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-fsanitize=undefined", "-fsanitize-undefined-trap-on-error",
                         "-I", os.path.join(ROOT, "paper_2607_16213_gb300", "csrc"),
                         os.path.join(ROOT, "tests", "c", "tree_fixed.cpp"), "-o", str(exe)], capture_output=True, text=True)
    assert cc.returncode == 0, cc.stderr
    run = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert run.returncode == 0 and run.stdout.strip() == "done", (run.returncode, run.stdout + run.stderr)
