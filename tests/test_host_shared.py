"""Plans of attention for batches that share cells (host C++, no GPU): compiles the planner together with a program that counts what plans hold, and runs it."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2605_26289_amd", "csrc")


@pytest.mark.parametrize("sanitizer", [None, "address,undefined"])
def test_every_row_meets_every_position_once_and_every_piece_is_joined(tmp_path, sanitizer):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no host C++ compiler")
    exe = str(tmp_path / "plan_shared_check")
    flags = [f"-fsanitize={sanitizer}"] if sanitizer else []
    cmd = [cxx, "-std=c++17", "-O1", "-g", "-pthread", *flags, os.path.join(ROOT, "tests", "plan_shared_check.cpp"),
           os.path.join(CSRC, "plan_shared.cpp"), os.path.join(CSRC, "pool.cpp"), "-o", exe]
    built = subprocess.run(cmd, capture_output=True, text=True)
    if built.returncode != 0 and sanitizer and "cannot find" in built.stderr.lower():
        pytest.skip("sanitizer runtime not installed")
    assert built.returncode == 0, built.stderr[-3000:]
    run = subprocess.run([exe, "400"], capture_output=True, text=True, timeout=300)
    if run.returncode != 0 and sanitizer and "runtime does not come first" in run.stderr:
        pytest.skip("another preloaded library keeps the sanitizer runtime from loading first")
    assert run.returncode == 0 and run.stdout.startswith("ok"), (run.stdout[-3000:], run.stderr[-2000:])
