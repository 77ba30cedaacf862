"""What importing the package leaves alone: it counts no GPUs, so that a process can still fork children that use one, or settle
which GPUs it sees, before its first call."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _python(code: str) -> None:
    res = subprocess.run([sys.executable, "-c", code], cwd=ROOT, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)
    assert res.returncode == 0, res.stdout[-2000:]


def test_importing_asks_for_no_device():
    _python("import torch\n"
            "def asked(*a): raise AssertionError('a device was asked for')\n"
            "torch.cuda.device_count = torch.cuda.current_device = torch._C._cuda_getDeviceCount = asked\n"
            "import paper_2005_10761_amd\n"
            "assert not torch.cuda.is_initialized()")


def test_a_child_forked_after_the_import_may_use_a_gpu():
    # (without amdsmi torch counts GPUs by the runtime, which a forked child cannot use any more)
    _python("import os, torch\n"
            "torch.cuda._device_count_amdsmi = lambda: -1\n"
            "import paper_2005_10761_amd\n"
            "child = os.fork()\n"
            "if child == 0: os._exit(int(torch.cuda._is_in_bad_fork()))\n"
            "assert os.waitstatus_to_exitcode(os.waitpid(child, 0)[1]) == 0")


@pytest.mark.gpu
def test_a_gpu_that_is_seen_after_the_import_only():
    _python("import torch\n"
            "count, torch.cuda.device_count = torch.cuda.device_count, lambda: 0\n"
            "import paper_2005_10761_amd as rt\n"
            "torch.cuda.device_count = count\n"
            "x = torch.arange(6.0, device='cuda').reshape(2, 3)\n"
            "out = torch.empty_like(x)\n"
            "rt.dropout(x, out, 0.0, 1, 2)\n"
            "assert torch.equal(out, x)")
