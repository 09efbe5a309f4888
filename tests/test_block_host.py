"""What attention over pages does on the host where there is no GPU: importing the binding."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_binding_imports_with_a_torch_without_gpu_support():
    """Such a torch has no _cuda_* names in torch._C."""
    code = ("import torch\n"
            "for n in [n for n in dir(torch._C) if n.startswith('_cuda_')]: delattr(torch._C, n)\n"
            "from paper_2604_18348_amd import binding\n"
            "assert binding.BlockParams(B=1, Hq=1, Hkv=1, d=64).blocks == 1\n")
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
