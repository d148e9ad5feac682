"""The binding of the microscaled 4-bit entry points without a GPU."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_training_needs_no_private_name_of_torch():
    """The network module imports where torch does not give the current stream as a number."""
    code = ("import torch\n"
            "if hasattr(torch._C, '_cuda_getCurrentRawStream'): del torch._C._cuda_getCurrentRawStream\n"
            "from paper_2106_05373_amd import mx, pipeline\n"
            "class Current:\n"
            "    def __init__(self, device): self.cuda_stream = 100 + device\n"
            "torch.cuda.current_stream = Current\n"
            "assert mx._raw_stream(3) == 103\n")
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
