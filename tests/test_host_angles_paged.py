"""Which angle turns a channel of a key on its way into the paged cache (csrc/lq_deal_paged.h), compiled for the host: an index
beyond a token's angles would be read beyond the LDS that holds them."""
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "..", "paper_2503_19950_amd", "csrc")


def test_every_channel_takes_an_angle_that_is_there(tmp_path):
    exe = tmp_path / "angles_paged"
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-Werror", "-I", CSRC, "-o", str(exe),
                    os.path.join(HERE, "host", "angles_paged.cpp")], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout + r.stderr
