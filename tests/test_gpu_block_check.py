"""GPU: the attention block's operators in the checking build (libfgq_check.so:
every buffer load and every store tested against its extent) and twice in the
normal one: no violation, and the same bytes every time."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import block_cases

fgq = pytest.importorskip("paper_1705_01462_amd")

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def first():
    return block_cases.run_cases(fgq, torch)


def test_checking_build_reports_no_violation(tmp_path, first):
    env = dict(os.environ, FGQ_LIBRARY="check")
    r = subprocess.run([sys.executable, "-u", os.path.join(ROOT, "tests", "block_cases.py"), str(tmp_path)],
                       env=env, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-3000:]
    assert "libfgq_check.so" in r.stdout
    n, site, off = (int(v) for v in open(tmp_path / "violations.txt").read().split())
    assert n == 0, f"{n} out-of-bounds accesses, the first at site {site}, offset {off}"
    assert len(first) > 100
    for k, v in first.items():
        got = np.load(tmp_path / (k + ".npy"))
        assert got.dtype == v.dtype and got.shape == v.shape and got.tobytes() == v.tobytes(), k


def test_repeated_runs_are_identical(first):
    again = block_cases.run_cases(fgq, torch)
    for k, v in first.items():
        assert again[k].tobytes() == v.tobytes(), k
