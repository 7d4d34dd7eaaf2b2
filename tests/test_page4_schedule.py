"""The work items of sekv_page_attend over 4-bit pages walked through on the host, built with g++ under the address and
undefined-behaviour sanitizers (tests/page4_checks.cpp), and that both kernels of a call plan it alike.  No GPU is involved."""

import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_31145_amd", "csrc")


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_items_cover_every_key_once(tmp_path):
    exe = tmp_path / "page4_checks"
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-Wall", "-Werror", "-fsanitize=address,undefined",
           "-fno-sanitize-recover=all", f"-I{CSRC}", os.path.join(ROOT, "tests", "page4_checks.cpp"), "-o", str(exe)]
    res = subprocess.run(cmd, capture_output=True, text=True, timeout=300)
    assert res.returncode == 0, res.stdout + res.stderr
    run = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0, run.stdout + run.stderr
    assert "all 4-bit page checks passed" in run.stdout


def test_both_kernels_of_a_call_plan_it_alike():
    """The join reads partials at the chunk borders at which the items wrote them."""
    with open(os.path.join(CSRC, "sekv_page_attend_inst.hip")) as f:
        plans = re.findall(r"Plan plan = (make_plan.*);", f.read())
    assert len(plans) == 2 and plans[0] == plans[1], plans
