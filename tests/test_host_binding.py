"""What the binding does before it calls the library.  No GPU needed."""
import types

import pytest
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


def test_tensors_of_other_dimensions_are_refused(monkeypatch):
    """A weight of four dimensions would have had its first matrix prepared alone; the others ended in errors of the language, not the call's."""
    monkeypatch.setattr(q, "_where", lambda t: t.get_device())
    bf16, u8 = torch.bfloat16, torch.uint8
    X, codes, scales, off = torch.zeros(4, 64, dtype=bf16), torch.zeros(4, 128, dtype=u8), torch.zeros(4, 8, dtype=u8), torch.tensor([0, 4])
    room = torch.zeros(384, 128, dtype=u8), torch.zeros(384, 8, dtype=u8)
    calls = [lambda: q.mx4_prepare_weight(torch.zeros(2, 2, 64, 48), *room, *room), lambda: q.mx4_prepare_weight(torch.zeros(64), *room, *room),
             lambda: q.mx4_quantize(X[0], codes, scales), lambda: q.mx4_quantize(X[None], codes, scales),
             lambda: q.mx4_dequantize(codes, scales, X[None]), lambda: q.check_group_offsets(None, 4, torch.zeros(1, dtype=torch.int32)),
             lambda: q.mx4_linear_fwd(X[0, 0], None, codes, scales, 64, 48, None, None, 0, 1.0, torch.zeros(4, 48), None),
             lambda: q.grouped_linear_fwd(X[0, 0], off, X[None], 1.0, X, None), lambda: q.grouped_linear_fwd(X, None, X[None], 1.0, X, None),
             lambda: q.grouped_linear_bwd_dw(X[None], X, off, 1.0, torch.zeros(1, 64, 64), None),
             lambda: q.grouped_linear_bwd_dw(X, X[0], off, 1.0, torch.zeros(1, 64, 64), None),
             lambda: q.grouped_linear_bwd_dw(X, X, None, 1.0, torch.zeros(1, 64, 64), None)]
    for i, call in enumerate(calls):
        with pytest.raises(q.QuaffError) as e:
            call()
        assert e.value.status == q.ERR_SHAPE, i
