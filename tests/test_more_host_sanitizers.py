"""The host side of the 4-bit products, layer norm and dropout (sizes, plans, refusals) under AddressSanitizer and
UndefinedBehaviorSanitizer, as a program of its own: host code only, no GPU is involved."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
DRIVER = os.path.join(ROOT, "tests", "host_sanitize", "more_driver.cpp")
SOURCES = ("rtopk_mx4.hip", "rtopk_norm.hip", "rtopk_dropout.hip")


def test_host_side_under_sanitizers(tmp_path):
    from paper_2005_10761_amd import build as hip_build
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not os.path.exists(hipcc) and shutil.which("hipcc") is None:
        pytest.skip("no hipcc")
    exe = str(tmp_path / "more_driver")
    flags = [f for f in hip_build.HIPCC_FLAGS if f not in ("-O3", "-fPIC", "-shared")]
    san = []
    for f in ("-fsanitize=address", "-fsanitize=undefined", "-fno-sanitize-recover=undefined"):
        san += ["-Xarch_host", f]                 # host code only
    cmd = [hipcc, "-O1", "-g"] + flags + san + ["-o", exe, DRIVER] + [f for f in hip_build.sources() if os.path.basename(f) in SOURCES]
    res = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert res.returncode == 0, res.stdout[-4000:]
    env = dict(os.environ, ASAN_OPTIONS="abort_on_error=0:halt_on_error=1:detect_leaks=0",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    res = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, env=env, timeout=300)
    assert res.returncode == 0, res.stdout[-4000:]
    assert "runtime error" not in res.stdout and "AddressSanitizer" not in res.stdout, res.stdout[-4000:]
    assert ", 0 failures" in res.stdout, res.stdout[-2000:]
