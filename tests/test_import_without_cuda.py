"""The package under a torch that was built without CUDA (CPU only)."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_package_imports_under_a_torch_without_cuda():
    """The closed forms run on the host: neither they nor the import need a torch that was built with CUDA."""
    code = ("import torch\n"
            "for name in [n for n in dir(torch._C) if n.startswith('_cuda_')]:\n"
            "    delattr(torch._C, name)\n"
            "import paper_2609_34370_b200 as spx\n"
            "print(spx.selective_batch(8.0, 2, 0.25))\n")
    run = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True)
    assert run.returncode == 0, run.stderr
    assert run.stdout.strip()
