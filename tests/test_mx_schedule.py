"""The product's tile and division of K (csrc/mx_schedule.h), which fix the order of its sums: a function of the shape alone,
checked on the host.  No GPU needed."""
import os
import re
import subprocess

ROOT = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..")
CSRC = os.path.join(ROOT, "paper_2205_03494_b200", "csrc")


def test_schedules_keep_what_the_kernels_rely_on(tmp_path):
    exe = str(tmp_path / "mx_schedule_check")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-o", exe, os.path.join(ROOT, "tests", "host", "mx_schedule_check.cpp")])
    run = subprocess.run([exe], capture_output=True, text=True)
    assert run.returncode == 0, run.stdout


def test_the_device_decides_nothing_but_the_grid():
    """The count of the device's SMs is asked for in one place of the product: how many CTAs walk over the tiles."""
    source = open(os.path.join(CSRC, "omc_mx_matmul.cu")).read()
    assert len(re.findall(r"sm_count\(\)", source)) == 1
    assert "sm_count" not in open(os.path.join(CSRC, "mx_schedule.h")).read()
