"""The binding's choice of a stream, without a GPU."""
import types

import torch

from paper_2609_09095_b200 import binding


def test_current_stream_by_the_public_form(monkeypatch):
    """A torch without the private shortcut to the current stream's handle: the stream object's own."""
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: types.SimpleNamespace(cuda_stream=0x1234))
    assert binding._stream(None) == 0x1234


def test_given_streams():
    assert binding._stream(0) == 0 and binding._stream(7) == 7
    assert binding._stream(types.SimpleNamespace(cuda_stream=9)) == 9
