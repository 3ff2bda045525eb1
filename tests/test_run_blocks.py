"""The reads of rows that start anywhere, enumerated on the host over widths, rows
and addresses (tests/c/test_run_blocks.cpp): inside their array, and complete."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_runs_are_read_inside_their_arrays(tmp_path):
    exe = os.path.join(str(tmp_path), "test_run_blocks")
    cmd = ["g++", "-std=c++17", "-O2", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2106_08846_gb300", "csrc"), "-o", exe,
           os.path.join(ROOT, "tests", "c", "test_run_blocks.cpp")]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "all runs inside" in r.stdout
