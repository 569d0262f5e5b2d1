"""How many clusters of a kernel fit is a number of each device, and a query that failed is no answer:
neither may be kept for the process."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2202_11836_gb300", "csrc")


def test_count_per_device(tmp_path):
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    exe = tmp_path / "device_count"
    r = subprocess.run([cxx, "-std=c++17", "-Wall", "-Wextra", "-Werror", "-pthread", "-I", CSRC,
                        os.path.join(ROOT, "tests", "c", "device_count.cpp"), "-o", str(exe)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout


def test_no_occupancy_kept_for_the_process():
    """A function's static number: an initializer that asks the device, or a lambda that may."""
    for f in sorted(os.listdir(CSRC)):
        src = open(os.path.join(CSRC, f)).read()
        if "Occupancy" in src or "at_once" in src:
            found = re.search(r"\bstatic (const )?int \w+(\[\w*\])? *= *(\[&\]|\{? *\w*(at_once|Occupancy)\w*\()", src)
            assert not found, (f, found.group())
