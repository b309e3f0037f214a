"""The bytes that the norm kernels' row copies read (csrc/row_copy.h), checked on the host: no GPU needed."""
import os
import subprocess

ROOT = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..")


def test_rows_are_read_whole_and_nothing_else_is(tmp_path):
    exe = str(tmp_path / "row_copy_check")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-o", exe, os.path.join(ROOT, "tests", "host", "row_copy_check.cpp")])
    run = subprocess.run([exe], capture_output=True, text=True)
    assert run.returncode == 0, run.stdout
