"""Which kernel an 8-bit product takes (csrc/i8_schedule.h), a function of the shape alone, checked on the host.  No GPU needed."""
import os
import subprocess

ROOT = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..")


def test_schedules_keep_what_the_kernels_rely_on(tmp_path):
    exe = str(tmp_path / "byte_schedule_check")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-o", exe, os.path.join(ROOT, "tests", "host", "byte_schedule_check.cpp")])
    run = subprocess.run([exe], capture_output=True, text=True)
    assert run.returncode == 0, run.stdout
