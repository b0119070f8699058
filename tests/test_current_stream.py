"""The stream that a call takes when it is given none: torch's current one, by whichever name torch has for it."""
import os
import subprocess
import sys

import pytest
import torch

import paper_2409_12517_amd as ssg

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_without_torchs_private_name():
    code = """
import types, torch
if hasattr(torch._C, "_cuda_getCurrentRawStream"):
    del torch._C._cuda_getCurrentRawStream
torch.cuda.current_device = lambda: 0
torch.cuda.current_stream = lambda: types.SimpleNamespace(cuda_stream=77)
import paper_2409_12517_amd as ssg
print(ssg._stream(None), ssg._stream(5), ssg._stream(types.SimpleNamespace(cuda_stream=6)))
"""
    out = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert out.returncode == 0, out.stderr
    assert out.stdout.split() == ["77", "5", "6"]


@pytest.mark.gpu
def test_is_torchs_current_stream():
    assert ssg._stream(None) == torch.cuda.current_stream().cuda_stream
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        assert ssg._stream(None) == side.cuda_stream != 0
    assert ssg._stream(None) == torch.cuda.current_stream().cuda_stream
