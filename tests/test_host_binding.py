"""What the binding does before it calls the library.  No GPU needed."""
import types

import torch

from paper_2505_14742_amd import binding as q


def test_the_stream_comes_from_public_names_where_torch_has_no_raw_accessor(monkeypatch):
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream")
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: types.SimpleNamespace(cuda_stream=77))
    assert q._stream() == 77


def test_the_raw_accessor_is_asked_for_the_current_device(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 100 + device)
    assert q._stream() == 103
