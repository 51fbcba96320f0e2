"""What the gated recurrence, the turned heads and the orthogonalised updates launch, over their sizes, on the CPU: their host side with a
stand-in for the runtime, which checks every launch against the limits of one (threads, workgroups, LDS and the leave to have more than
64 KB of it)."""
import os
import subprocess

from paper_2502_00021_amd import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_every_launch_is_one_that_the_device_takes(tmp_path):
    flags = [f for f in build.HIPFLAGS if f != "-shared" and not f.startswith("-W")]
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    sources = [os.path.join(build.CSRC, f) for f in ("layer_norm.hip", "linear_attention.hip", "gated_recurrence.hip", "head_norm.hip", "orthogonalise.hip", "learner_api.cpp")]
    sources.append(os.path.join(ROOT, "tests", "operator_launch_check_main.cpp"))
    objects = [str(tmp_path / (os.path.basename(s) + ".o")) for s in sources]
    jobs = [subprocess.Popen([hipcc, *flags, "-w", "--cuda-host-only", "-I", os.path.join(ROOT, "include"), "-I", build.CSRC, "-I", os.path.join(ROOT, "tests"), "-c", s, "-o", o],
                             stderr=subprocess.PIPE, text=True) for s, o in zip(sources, objects)]
    for job in jobs:
        err = job.communicate()[1]
        assert job.returncode == 0, err[-2000:]
    exe = str(tmp_path / "launch_check")
    # (the device code that the objects name is not there: nothing looks at it)
    subprocess.check_call(["g++", *objects, "-Wl,--unresolved-symbols=ignore-all", "-o", exe])
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-1000:]
    launches, kernels, large = (int(x) for x in r.stdout.split()[1:])
    assert launches > 20000 and kernels > 50 and large > 100, r.stdout
