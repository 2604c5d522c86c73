"""Waits of the product's kernels that run out (tests/q8_timeout_run.py, in a process with the checked build of the library)."""
import os
import subprocess
import sys

import pytest

from paper_2309_06973_b200 import build as build_mod

pytestmark = pytest.mark.gpu
HERE = os.path.dirname(os.path.abspath(__file__))


def test_waits_that_run_out():
    lib = build_mod.build(checked=True)
    out = subprocess.run([sys.executable, os.path.join(HERE, "q8_timeout_run.py")], env=dict(os.environ, DNNS_LIBRARY=lib),
                         capture_output=True, text=True, timeout=600)
    assert out.returncode == 0, out.stdout[-2000:] + out.stderr[-2000:]
    assert out.stdout.strip().splitlines()[-1].startswith("ok"), out.stdout[-500:]
