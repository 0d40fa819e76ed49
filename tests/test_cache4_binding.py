"""The binding of the 4-bit cache without a GPU."""

import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _python(code):
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    return r.stdout


def test_import_without_the_raw_stream_call():
    """torch._C._cuda_getCurrentRawStream is not public: without it the binding asks the public call."""
    out = _python("import torch\n"
                  "if hasattr(torch._C, '_cuda_getCurrentRawStream'): del torch._C._cuda_getCurrentRawStream\n"
                  "from paper_2608_08086_amd import archer\n"
                  "class S: cuda_stream = 77\n"
                  "torch.cuda.current_stream = lambda dev: S if dev == 3 else None\n"
                  "print(archer._raw_stream(3))")
    assert out.split()[-1] == "77"
