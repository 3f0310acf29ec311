"""Which stream a call without one goes to: torch's current stream, as its handle."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_default_stream_argument_is_the_current_stream(K):
    assert K._stream(None) == torch.cuda.current_stream().cuda_stream
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        assert K._stream(None) == s.cuda_stream == torch.cuda.current_stream().cuda_stream
    assert K._stream(s) == s.cuda_stream and K._stream(7) == 7
    assert K._stream(None) == torch.cuda.current_stream().cuda_stream
