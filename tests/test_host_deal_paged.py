"""Plans of attention over the paged cache and the arithmetic of its places (csrc/lq_plan_paged.h, lq_deal_paged.h), compiled for
the host and run over random batches.  A unit that is left out would drop tokens, a partial result or a page out of place would be
read or written beyond its buffer."""
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "..", "paper_2503_19950_amd", "csrc")


def test_every_unit_is_taken_once_and_places_stay_inside(tmp_path):
    exe = tmp_path / "deal_paged"
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-Werror", "-I", CSRC, "-o", str(exe),
                    os.path.join(HERE, "host", "deal_paged.cpp")], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr
