"""The state that a tile of a long recurrence begins with does not depend on which of the tiles before it had published their states (see
stretches_check.cpp)."""
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


def test_the_same_bits_whatever_was_published_first(tmp_path):
    if shutil.which("g++") is None:
        pytest.skip("no g++")
    exe = str(tmp_path / "stretches_check")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-ffp-contract=off", "-o", exe, os.path.join(HERE, "stretches_check.cpp")], check=True)
    run = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert run.returncode == 0 and "stretches_check ok" in run.stdout, run.stdout + run.stderr
