"""The batched serving calls' launches (CPU): tests/c_consumer/batch_launches.cpp takes the place of
the runtime's launch functions, calls the entry points and checks the grids that they ask for."""

import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
PKG = os.path.join(ROOT, "paper_2609_33503_amd")
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")


@pytest.fixture(scope="module")
def driver(rk, tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("needs a host C++ compiler")
    exe = str(tmp_path_factory.mktemp("launches") / "batch_launches")
    cmd = ["g++", "-std=c++17", "-O2", "-Wall", "-Wextra", "-D__HIP_PLATFORM_AMD__",
           "-isystem", os.path.join(ROCM, "include"), "-I", os.path.join(ROOT, "include"),
           "-I", os.path.join(PKG, "csrc"), os.path.join(HERE, "c_consumer", "batch_launches.cpp"),
           "-o", exe, "-rdynamic", "-L", PKG, "-lrelaxkv", "-Wl,-rpath," + PKG,
           "-L", os.path.join(ROCM, "lib"), "-lamdhip64", "-Wl,-rpath," + os.path.join(ROCM, "lib")]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    return exe


def _run(exe, *args):
    r = subprocess.run([exe, *args], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.startswith("ok "), r.stdout + r.stderr[-4000:]


def test_every_workgroup_and_partial_row_of_a_step(driver):
    """Random steps: all workgroups of the plan's split are launched, all partial rows have room
    (about one float32 step in 300 has more splits than 256 workgroups and three per item)."""
    _run(driver, "steps", "300000")


def test_launches_of_the_largest_fresh_rows(driver):
    _run(driver, "fresh")


def test_launches_of_the_largest_batches(driver):
    _run(driver, "batch")


def test_launches_of_the_selection(driver):
    _run(driver, "select")
