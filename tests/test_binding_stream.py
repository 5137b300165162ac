"""The current stream as the operators' calls find it (no GPU needed: torch's own functions are stood in for)."""
from types import SimpleNamespace

import torch

from paper_1804_04512_amd import binding as B


def test_with_and_without_the_short_way(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda index=None: SimpleNamespace(device=torch.device("cuda", 3), cuda_stream=0x1230))
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 0x4560 + index, raising=False)
    assert B._call_stream(None) == (torch.device("cuda", 3), 0x4563)
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream")
    assert B._call_stream(None) == (torch.device("cuda", 3), 0x1230)
