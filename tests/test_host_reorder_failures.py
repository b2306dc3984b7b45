"""dk_seq_reorder's bookkeeping where something goes wrong on the way (host C++, no GPU)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def run_check(tmp_path, what, sanitizer):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no host C++ compiler")
    exe = str(tmp_path / "reorder_failures")
    flags = [f"-fsanitize={sanitizer}"] if sanitizer else []
    cmd = [cxx, "-std=c++17", "-O1", "-g", "-pthread", *flags, os.path.join(ROOT, "tests", "reorder_failures.cpp"),
           os.path.join(ROOT, "paper_2605_26289_amd", "csrc", "pool.cpp"), "-o", exe]
    built = subprocess.run(cmd, capture_output=True, text=True)
    if built.returncode != 0 and sanitizer and "cannot find" in built.stderr.lower():
        pytest.skip("sanitizer runtime not installed")
    assert built.returncode == 0, built.stderr[-3000:]
    run = subprocess.run([exe, what], capture_output=True, text=True, timeout=120)
    if run.returncode != 0 and sanitizer and "runtime does not come first" in run.stderr:
        pytest.skip("another preloaded library keeps the sanitizer runtime from loading first")
    assert run.returncode == 0 and run.stdout.startswith("ok"), (run.stdout[-2000:], run.stderr[-2000:])


@pytest.mark.parametrize("sanitizer", [None, "address,undefined"])
def test_a_failed_allocation_loses_no_granule(tmp_path, sanitizer):
    run_check(tmp_path, "granules", sanitizer)


@pytest.mark.parametrize("sanitizer", [None, "address,undefined"])
def test_giving_cells_back_needs_no_memory(tmp_path, sanitizer):
    run_check(tmp_path, "giving_back", sanitizer)


@pytest.mark.parametrize("sanitizer", [None, "address,undefined"])
def test_a_failed_allocation_leaves_every_slot_as_it_was(tmp_path, sanitizer):
    run_check(tmp_path, "out_of_memory", sanitizer)


@pytest.mark.parametrize("sanitizer", [None, "address,undefined", "thread"])
def test_no_other_call_comes_between_a_reorder_and_its_end(tmp_path, sanitizer):
    run_check(tmp_path, "one_step", sanitizer)


@pytest.mark.parametrize("sanitizer", ["thread", "address,undefined"])
def test_searches_on_several_threads(tmp_path, sanitizer):
    run_check(tmp_path, "threads", sanitizer)


@pytest.mark.parametrize("sanitizer", [None, "address,undefined"])
def test_cells_that_no_slot_sees_come_back(tmp_path, sanitizer):
    run_check(tmp_path, "cells_come_back", sanitizer)


@pytest.mark.parametrize("sanitizer", [None, "address,undefined"])
def test_long_chains_are_let_go_of(tmp_path, sanitizer):
    run_check(tmp_path, "long_chains", sanitizer)
