"""The stream that a call without one goes to: torch's current one, by whichever call this torch has."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = """
import types, torch
if hasattr(torch._C, "_cuda_getCurrentRawStream"):
    del torch._C._cuda_getCurrentRawStream
torch.cuda.current_stream = lambda *a: types.SimpleNamespace(cuda_stream=77)
torch.cuda.current_device = lambda: 0
from paper_2606_23406_amd import hq
assert hq._stream_handle() == 77
assert hq._stream_handle(types.SimpleNamespace(cuda_stream=5)) == 5
print("ok")
"""


def test_a_torch_without_the_raw_handle():
    r = subprocess.run([sys.executable, "-c", PROGRAM], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.stdout == "ok\n", r.stderr[-500:]


@pytest.mark.gpu
def test_the_handle_is_the_current_streams(monkeypatch):
    import torch
    from paper_2606_23406_amd import hq
    side = torch.cuda.Stream()
    for raw in (hq._raw_stream, None):
        monkeypatch.setattr(hq, "_raw_stream", raw)
        assert hq._stream_handle() == torch.cuda.current_stream().cuda_stream
        with torch.cuda.stream(side):
            assert hq._stream_handle() == side.cuda_stream
        assert hq._stream_handle(side) == side.cuda_stream != hq._stream_handle()
