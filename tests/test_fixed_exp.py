"""The fixed-point weights of the sampling kernels, run on the host: how far
they are from exp, and that they never rise where scores fall."""
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2609_18703_gb300", "csrc")


@pytest.mark.skipif(shutil.which("g++") is None, reason="no host compiler")
def test_weights_are_exp_to_forty_bits(tmp_path):
    exe = str(tmp_path / "model")
    subprocess.run([shutil.which("g++"), "-std=c++17", "-O1", "-ffp-contract=off", "-I", CSRC,
                    os.path.join(HERE, "fixed_exp_model.cpp"), "-o", exe], check=True)
    worst, risen, one, none = subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split()
    # pairs of floats: some 2^-44 for the argument, the table and each of the terms
    assert float(worst) < 2.0
    assert (risen, one, none) == ("0", "1", "1")
