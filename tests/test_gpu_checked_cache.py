"""The bounds-checked build (OCCAM_CHECKED=1) on the cache operators' own tests: every computed row,
page, table column, list place, keep flag and partial result is tested in-kernel (check.cuh), and nothing
is recorded. The checked library is built on demand and loaded in a process of its own."""

from __future__ import annotations

import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_checked_build_of_the_cache_operators():
    from paper_2605_29657_gb300 import build as pb

    pb.build(checked=True)
    r = subprocess.run([sys.executable, os.path.join(ROOT, "tests", "_checked_cache_cases.py")], cwd=ROOT,
                       capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-4000:]
    assert "done 34" in r.stdout, r.stdout
