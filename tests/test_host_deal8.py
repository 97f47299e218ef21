"""Plans of attention over the 8-bit cache: the host's planner and the kernel's own arithmetic (csrc/lq_plan8.h, lq_deal8.h),
compiled for the host and run over random batches.  A unit that is left out would drop tokens, a partial result out of place
would be written beyond the workspace."""
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "..", "paper_2503_19950_amd", "csrc")


def test_every_unit_is_taken_once_and_partial_results_have_room(tmp_path):
    exe = tmp_path / "deal8"
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-Werror", "-I", CSRC, "-o", str(exe),
                    os.path.join(HERE, "host", "deal8.cpp")], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr
