"""How heads are dealt to lanes: for every head, rotated part, type and direction each lane reads inside a token's row of the tables, and every channel has
one owner.  The arithmetic is the kernel's own, compiled for the host.  No GPU needed."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_lanes_stay_inside_the_tables(tmp_path):
    exe = str(tmp_path / "qk_lanes")
    build = subprocess.run(["g++", "-std=c++17", "-O2", "-D__host__=", "-D__device__=", "-D__forceinline__=inline",
                            "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2512_05746_amd", "csrc"),
                            os.path.join(ROOT, "tests", "qk_lanes_driver.cpp"), "-o", exe],
                           stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert build.returncode == 0, build.stdout
    run = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=120)
    assert run.returncode == 0, run.stdout
