"""The binding of the 4-bit cache without a GPU."""

import os
import subprocess
import sys

import pytest
import torch

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


@pytest.mark.parametrize("name", ["max_cached", "fresh_stride", "slot_rows", "page_size", "cache page_size", "head_dim"])
@pytest.mark.parametrize("value", [2**31, 2**32, 2**32 + 64, -2**31 - 1])
def test_host_integers_beyond_32_bits(name, value, monkeypatch):
    """They would reach the library as their low 32 bits: a max_cached of 2^32 as 0, every key left out."""
    from paper_2608_08086_amd import archer as a
    # host tensors in the place of the device's: every refusal comes before a launch
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)
    for f in ("archer_cache4_plan", "archer_op_attention_cache4"):
        monkeypatch.setattr(a.lib, f, lambda *x: pytest.fail("the library was called"))
    i = lambda *x: torch.tensor(x, dtype=torch.int32)  # noqa: E731
    data = torch.zeros(4, 2, 64 * 136, dtype=torch.uint8)
    h = torch.zeros(2, 2, 128, dtype=torch.float16)
    with pytest.raises(a.ArcherError, match=name.split()[-1] + ".*32 bits"):
        if name in ("slot_rows", "page_size"):
            kw = dict(page_size=64, slot_rows=4)
            kw[name] = value
            a.cache4_plan(i(0), i(1), table=i(0, 0)[None], free_pages=i(0), pool=i(0, 1), **kw)
        elif name in ("cache page_size", "head_dim"):
            kw = dict(page_size=64, head_dim=128)
            kw[name.split()[-1]] = value
            a.Cache4(data, **kw)
        else:
            kw = dict(max_cached=9, fresh_stride=8)
            kw[name] = value
            a.op_attention_cache4(h, a.Cache4(data, 64, 128), i(0, 1)[:, None], i(1, 1), **kw)
