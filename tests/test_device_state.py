"""What the library remembers per device: a kernel's LDS limit and the number of compute units
(csrc/sq_internal.h against a runtime that only counts; no GPU)."""

import os
import subprocess

from paper_2405_16406_amd import build

HERE = os.path.dirname(os.path.abspath(__file__))


def test_limits_and_units_are_kept_for_each_device(tmp_path):
    out = str(tmp_path / "state")
    r = subprocess.run([build.hipcc(), *build.COMMON, f"--offload-arch={build.ARCH}", os.path.join(HERE, "device_state_host.cpp"),
                        "-o", out], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([out], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stderr
    rows = [tuple(int(x) for x in line.split()) for line in r.stdout.splitlines()]
    # a failure (1: invalid value) is tried again; a second device, and a second kernel, has its own limit;
    # devices beyond the table are set each time
    assert rows[:10] == [(1, 1), (2, 0), (2, 0), (3, 0), (3, 0), (3, 0), (4, 0), (5, 0), (6, 0), (7, 0)]
    assert rows[10:] == [(1, 100, 0), (2, 101, 0), (2, 101, 0), (2, 100, 0), (3, 102, 0)]
