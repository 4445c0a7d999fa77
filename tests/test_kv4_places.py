"""Where the calls on a 4-bit cache look: groups of tokens, pages, tiles and parts, for arrays on the device that say sensible things and for arrays that
do not.  The arithmetic is the kernels' own, compiled for the host.  No GPU needed."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_places_stay_inside_the_call_and_the_cache(tmp_path):
    exe = str(tmp_path / "kv4_places")
    build = subprocess.run(["g++", "-std=c++17", "-O2", "-fsanitize=undefined", "-fno-sanitize-recover", "-D__host__=", "-D__device__=", "-D__forceinline__=inline",
                            "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2512_05746_amd", "csrc"),
                            os.path.join(ROOT, "tests", "kv4_places_driver.cpp"), "-o", exe],
                           stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert build.returncode == 0, build.stdout
    run = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=120)
    assert run.returncode == 0, run.stdout
