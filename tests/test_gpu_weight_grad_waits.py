"""What the weight gradient leaves behind where a wait inside its kernel runs out."""
import os
import subprocess
import sys

import pytest


@pytest.mark.gpu
def test_a_wait_that_runs_out_leaves_nans_and_nothing_else():
    program = os.path.join(os.path.dirname(os.path.abspath(__file__)), "weight_grad_waits.py")
    done = subprocess.run([sys.executable, program], capture_output=True, text=True, timeout=300)
    assert done.returncode == 0 and done.stdout.count("ok") == 16, done.stdout + done.stderr
