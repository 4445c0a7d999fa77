"""Whether two strided views share memory, as the checks of result buffers decide it: against marking every byte.  The arithmetic is the
binding's own, in a program of its own.  No GPU needed."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_shared_memory_of_views(tmp_path):
    exe = str(tmp_path / "overlap")
    build = subprocess.run(["g++", "-std=c++17", "-O2", "-I", os.path.join(ROOT, "paper_2512_05746_amd", "csrc"),
                            os.path.join(ROOT, "tests", "overlap_driver.cpp"), "-o", exe],
                           stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert build.returncode == 0, build.stdout
    run = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=120)
    assert run.returncode == 0, run.stdout
