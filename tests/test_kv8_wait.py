"""The bounded waits of the 8-bit cache's tcgen05 kernel run out (no fault, no hang): the waiter that reaches its limit
gives up, the CTA's other waiters are released, and the status is recorded once."""
import os
import subprocess

import pytest

from paper_2402_02082_gb300 import build

HERE = os.path.dirname(os.path.abspath(__file__))
pytestmark = pytest.mark.gpu


def test_wait_runs_out(tmp_path):
    exe = str(tmp_path / "wait_check")
    cmd = [build.nvcc(), *build.ARCH, "-std=c++17", "-O3", "--expt-relaxed-constexpr", "-I", build.CSRC,
           "-I", build.INCLUDE, os.path.join(HERE, "kv8_wait_check.cu"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout + r.stderr
    limit, released, done, idle, again, late, status, *us = (int(x) for x in r.stdout.split())
    assert (limit, released, done, idle) == (0, 0, 1, 2)  # gave up, released, completed, did not wait
    assert (again, late) == (1, 0)                        # with the flag set: a completed phase is seen, another not waited for
    assert status == 4                                    # kStatusTimeout: a wait that ran out
    assert 990000 <= us[0] <= 1200000                     # the limit of a second
    assert us[1] <= 1300000                               # by the flag: its own limit would have ended half a second later
    assert us[2] <= 50000
    assert us[4] <= 1350000 and us[5] <= 1350000          # asked again after all that, and not for another second
