"""The inner step's module imports under a torch that lacks the short ways to the current stream and device."""
import subprocess
import sys

from conftest import ROOT


def test_import_without_private_names():
    code = ("import torch\n"
            "for name in ('_cuda_getCurrentRawStream', '_cuda_getDevice'):\n"
            "    if hasattr(torch._C, name):\n"
            "        delattr(torch._C, name)\n"
            "from paper_2607_03011_gb300 import inner\n"
            "print(callable(inner.embed))\n")
    out = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True)
    assert out.returncode == 0, out.stderr
    assert out.stdout.strip() == "True"
