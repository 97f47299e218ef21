"""Limits of the plans of attention over the 8-bit cache (csrc/lq_plan8.h), compiled for the host: kernels that are built and room that a
workspace has are what random batches can ask for."""
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "..", "paper_2503_19950_amd", "csrc")


def test_plans_stay_within_what_is_built_and_allotted(tmp_path):
    exe = tmp_path / "plan8_limits"
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-Werror", "-I", CSRC, "-o", str(exe),
                    os.path.join(HERE, "host", "plan8_limits.cpp")], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr
