"""The size of a thread-block cluster is chosen, and allowed, on the device of the call: a host program with a stand-in for the CUDA runtime that has several devices."""
import os
import re
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2410_01518_b200", "csrc")


@pytest.mark.skipif(not shutil.which(os.environ.get("NVCC", "nvcc")), reason="no nvcc on this machine")
def test_every_device_and_every_size_of_shared_memory_is_asked_for_itself(tmp_path):
    program = str(tmp_path / "cluster_choice")
    subprocess.check_call([os.environ.get("NVCC", "nvcc"), "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-cudart", "none", "-I", CSRC,
                           os.path.join(HERE, "cluster_choice.cu"), os.path.join(HERE, "fake_cudart.cpp"), "-o", program])
    out = subprocess.run([program], capture_output=True, text=True, check=True).stdout
    calls = [tuple(map(int, m)) for m in re.findall(r"call device (\d+) items \d+ smem (\d+) cluster (\d+) status (\d+)", out)]
    assert calls == [(0, 50000, 16, 0), (1, 50000, 12, 0), (0, 50000, 16, 0), (1, 50000, 12, 0), (70, 50000, 16, 0), (1, 50000, 12, 0),
                     (0, 120000, 12, 0), (0, 50000, 16, 0), (0, 50000, 16, 0), (1, 50000, 12, 0)], out
    assert "refused" not in out
    # answers are kept: each device's question is asked once as long as the shared memory stays the same
    asked = re.findall(r"asked device (0|1) cluster (\d+) smem 50000", out.split("smem 120000")[0])
    assert len(asked) == len(set(asked)), out
