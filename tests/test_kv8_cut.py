"""How attention over the 8-bit cache is cut up (csrc/kv8_cut.h), evaluated on the host.  CPU only."""
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2606_21712_amd", "csrc")

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")


def test_steps(tmp_path):
    """Every token that a row sees is in one step of one part; no step begins in a page that the sequence does not have."""
    exe = str(tmp_path / "kv8_cut")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", CSRC, os.path.join(HERE, "native", "kv8_cut.cpp"),
                    "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True)
    assert r.returncode == 0 and "ok" in r.stdout, r.stderr
