"""Rows of a paged cache against their definition, on the CPU: nothing leaves the pool, whatever the table says."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_rows_stay_inside_of_the_pool(tmp_path):
    exe = tmp_path / "page_row_check"
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Wextra", "-I",
                    os.path.join(ROOT, "paper_2502_14317_amd", "csrc"), os.path.join(ROOT, "tests", "host", "page_row_check.cpp"), "-o", str(exe)],
                   check=True)
    done = subprocess.run([str(exe)], capture_output=True, text=True)
    assert done.returncode == 0 and done.stdout.strip() == "ok", done.stdout + done.stderr
