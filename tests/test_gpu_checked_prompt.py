"""The bounds-checked build (OCCAM_CHECKED=1) on the tests of whole-prompt attention, its gradient, append with the
rotation and attention over shared pages: every computed row, page and partial result is tested in-kernel
(check.cuh), and nothing is recorded. The checked library is loaded in a process of its own."""

from __future__ import annotations

import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_checked_build_of_the_prompt_operators():
    from paper_2605_29657_gb300 import build as pb

    pb.build(checked=True)
    r = subprocess.run([sys.executable, os.path.join(ROOT, "tests", "_checked_prompt_cases.py")], cwd=ROOT,
                       capture_output=True, text=True, timeout=900)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-4000:]
    assert "done" in r.stdout.splitlines()[-1], r.stdout
