"""Every launch of the 4-bit products, layer norm and dropout has a shape that the device takes, the largest sizes among them: their host
side is linked with a launch that only looks at the shape. Host code only, no GPU is involved."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
DRIVER = os.path.join(ROOT, "tests", "host_launch", "launch_driver.cpp")
SOURCES = ("rtopk_mx4.hip", "rtopk_norm.hip", "rtopk_dropout.hip")


def test_every_launch_has_a_shape_that_the_device_takes(tmp_path):
    from paper_2005_10761_amd import build as hip_build
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not os.path.exists(hipcc) and shutil.which("hipcc") is None:
        pytest.skip("no hipcc")
    flags = [f for f in hip_build.HIPCC_FLAGS if f != "-shared"] + ["--offload-host-only", "-c", "-o"]
    objects = []
    for src in [f for f in hip_build.sources() if os.path.basename(f) in SOURCES] + [DRIVER]:
        objects.append(str(tmp_path / (os.path.basename(src) + ".o")))
        res = subprocess.run([hipcc] + flags + [objects[-1]] + (["-x", "hip"] if src == DRIVER else []) + [src], stdout=subprocess.PIPE,
                             stderr=subprocess.STDOUT, text=True)
        assert res.returncode == 0, res.stdout[-4000:]
    exe = str(tmp_path / "launch_driver")
    # (there are no kernels to be registered: the symbol of their code stays unresolved)
    res = subprocess.run([shutil.which("g++") or "c++", "-no-pie", "-o", exe] + objects + ["-Wl,--unresolved-symbols=ignore-all"],
                         stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert res.returncode == 0, res.stdout[-4000:]
    res = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)
    assert res.returncode == 0 and ", 0 failures" in res.stdout, res.stdout[-4000:]
