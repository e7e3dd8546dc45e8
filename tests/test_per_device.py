"""Kernel attributes belong to a device, so what has been set is kept for each device and only where it succeeded.
One GPU cannot show it; the table that the launchers share is plain C++ and is checked on the host."""
import os
import re
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2609_32869_gb300", "csrc")


def test_table(tmp_path):
    cxx = shutil.which("g++") or shutil.which("c++")
    if not cxx:
        pytest.skip("no host C++ compiler")
    exe = str(tmp_path / "per_device_check")
    subprocess.run([cxx, "-std=c++17", "-O1", "-pthread", "-I", CSRC, os.path.join(HERE, "per_device_check.cpp"), "-o", exe],
                   check=True, capture_output=True, text=True)
    r = subprocess.run([exe], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout == "0 violations\n", r.stdout


@pytest.mark.parametrize("name", ["wf_kv4_attn.cu", "wf_beam.cu", "wf_paged.cu"])
def test_the_beam_calls_keep_nothing_for_all_devices(name):
    """Every static of these calls' launchers is such a table."""
    src = re.sub(r"//.*", "", open(os.path.join(CSRC, name)).read())
    held = [m for m in re.findall(r"^ +static (?!constexpr|__device__)(?!_assert)([^;=({]+)", src, flags=re.M)]
    assert held and all(h.strip().startswith("PerDevice ") for h in held), held
