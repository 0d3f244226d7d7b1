"""The fixed-point weights of the sampling kernels, run on the host: as exact at
temperatures of any size, below the normal numbers too."""
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2609_18703_gb300", "csrc")


@pytest.mark.skipif(shutil.which("g++") is None, reason="no host compiler")
def test_weights_at_temperatures_of_any_size(tmp_path):
    exe = str(tmp_path / "model")
    subprocess.run([shutil.which("g++"), "-std=c++17", "-O1", "-ffp-contract=off", "-I", CSRC,
                    os.path.join(HERE, "fixed_exp_scales_model.cpp"), "-o", exe], check=True)
    worst, n = subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split()
    # pairs of floats: some 2^-44 for the argument, the table and each of the terms
    assert float(worst) < 2.0 and int(n) > 900_000
