"""The current stream's handle where torch lacks its short way to it (a private function) (no GPU)."""

from types import SimpleNamespace

import torch

from paper_2609_30846_amd import ipk


def test_the_current_stream_without_the_private_function(monkeypatch):
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream")
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda index: SimpleNamespace(cuda_stream=100 + index))
    assert ipk._stream_ptr(None) == 103 and ipk._stream_ptr(None, 5) == 105
    assert ipk._stream_ptr(SimpleNamespace(cuda_stream=7)) == 7


def test_the_private_function_is_used_where_it_is(monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 200 + index)
    assert ipk._stream_ptr(None, 1) == 201
