"""The steps that linear attention's scan kernels ask for (csrc/steps.h, plain arithmetic that the kernels share) on the CPU: no lane of any
kernel reads outside the view that it is given, whole chunks, last ones and single steps, and what is written to a tile
is the vector of its place."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_no_request_for_a_step_that_is_none(tmp_path):
    exe = str(tmp_path / "steps_check")
    subprocess.check_call(["g++", "-std=c++17", "-O2", "-Wall", "-Wextra", os.path.join(ROOT, "tests", "steps_check_main.cpp"), "-o", exe])
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout[-2000:]
    requests, kernels = (int(x) for x in r.stdout.split()[1:])
    assert kernels == 18 and requests > 10 ** 7, r.stdout
