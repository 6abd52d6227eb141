"""The stream that the binding hands to a call made without one."""
import types

import pytest
import torch

from paper_2609_34555_amd import pulse as P


def test_a_torch_without_the_raw_handle(monkeypatch):
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: types.SimpleNamespace(cuda_stream=4711))
    assert P._stream(None) == 4711
    assert P._stream(5) == 5 and P._stream(types.SimpleNamespace(cuda_stream=6)) == 6


@pytest.mark.gpu
def test_the_current_stream_is_taken():
    side = torch.cuda.Stream()
    assert P._stream(None) == torch.cuda.current_stream().cuda_stream
    with torch.cuda.stream(side):
        assert P._stream(None) == side.cuda_stream == P._stream(side) != 0
    assert P._stream(None) == torch.cuda.current_stream().cuda_stream
