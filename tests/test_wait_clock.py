"""The clock of waits that span work of any length, compiled with the host compiler and run."""
import os
import subprocess
import tempfile

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2604_08133_b200", "csrc")


def test_a_wait_runs_out_only_when_nothing_moves():
    src = os.path.join(ROOT, "tests", "cpp", "wait_clock_test.cpp")
    with tempfile.TemporaryDirectory() as tmp:
        exe = os.path.join(tmp, "wait_clock_test")
        subprocess.run(["g++", "-std=c++17", "-O1", "-I", CSRC, src, "-o", exe], check=True)
        r = subprocess.run([exe], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.strip().endswith("ok"), r.stdout + r.stderr


def test_the_adapted_projections_long_waits_use_it():
    """The masked-V warps stand in one wait through all blocks that need no mask, the epilogue through a tile's K loop:
    neither is bounded by a launch's length."""
    with open(os.path.join(CSRC, "adapter.cu")) as f:
        lines = [line for line in f if "ok = mbar" in line and ("ctl.vstart" in line or "ctl.tmem_full" in line)]
    assert len(lines) == 2 and all("mbar_spin_progress_warp" in line for line in lines), lines
