"""How the warps of the persistent kernels leave once a wait was given up: the rule, compiled for the CPU."""
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)


def test_warps_that_meet_leave_together(tmp_path):
    program = str(tmp_path / "check")
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    include = [os.path.join(os.path.dirname(os.path.dirname(nvcc)), "include"), os.path.join(ROOT, "paper_2609_34420_b200", "csrc")]
    subprocess.check_call(["g++", "-std=c++20", "-O1", "-w", "-pthread", *["-I" + x for x in include], os.path.join(HERE, "item_exit_check.cpp"), "-o", program])
    run = subprocess.run([program], capture_output=True, text=True, timeout=60)
    assert run.returncode == 0, run.stdout
