"""The bounds-checked build on the operators over paged caches: rows and summaries inside the pool, record slots and
segment parts inside the workspace, places inside a selection.  On valid inputs it reports nothing and its outputs are
the release build's bit for bit."""
import json
import os
import subprocess
import sys

import pytest

import paged_checked_run

pytestmark = pytest.mark.gpu
HERE = os.path.dirname(os.path.abspath(__file__))


def test_checked_build_runs_clean_and_matches_release(cuda_ok):
    from paper_2601_08670_gb300 import build
    build.build(checked=True)
    res = subprocess.run([sys.executable, os.path.join(HERE, "paged_checked_run.py")],
                         env=dict(os.environ, PCED_LIB="checked"), capture_output=True, text=True, timeout=600)
    assert res.returncode == 0, res.stderr[-3000:]
    checked = json.loads(res.stdout.strip().splitlines()[-1])
    assert len(checked) == len(paged_checked_run.CASES)
    assert checked == paged_checked_run.run_cases()
    assert all(c["status"] == 0 for c in checked)
