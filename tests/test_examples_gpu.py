"""The examples run from the command line."""

import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("args", [["--rows", "3", "--d", "512", "--vocab", "777"], ["--rows", "20", "--d", "1024", "--vocab", "4099"]])
def test_quantized_exit(args):
    r = subprocess.run([sys.executable, os.path.join(ROOT, "examples", "quantized_exit.py"), *args],
                       capture_output=True, text=True, cwd=ROOT, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "first state's candidates" in r.stdout and "loss" in r.stdout
