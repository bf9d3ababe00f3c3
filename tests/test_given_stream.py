"""Memory for calls that are given a stream: the helpers' arguments (test_given_stream_gpu.py has the streams)."""
import pytest
import torch

from paper_2505_19115_b200 import binding as nb


class Stream:
    cuda_stream = 0


def test_memory_on_a_given_stream_is_laid_out_as_asked():
    n, like = nb._native(), torch.zeros(1)
    for stream in (None, Stream):
        t = n.empty_on(stream, like, torch.bfloat16, 1, 3, 40)
        assert t.shape == (3, 40) and t.dtype == torch.bfloat16 and t.is_contiguous() and t.device == like.device
        assert n.empty_on(stream, like, torch.uint8, 0, 7).shape == (7,) and n.empty_on(stream, like, torch.float32, 1, 2, 3, 4).shape == (2, 3, 4)
        assert n.empty_rows(like, 4, 8, stream).shape == (4, 8)
        assert n.empty_fp8(like, 0, 130, 24, 1, 0, nb.SF_SWIZZLED, stream)[0].stride() == (32, 1)
        assert [t.shape for t in n.expert_buffers(like, 5, 2, 3, 256, stream)] == [(3,), (4,), (5, 2), (256,)]
    assert nb._empty((2, 3), torch.float32, like, Stream).shape == nb._empty((2, 3), torch.float32, like, None).shape == (2, 3)
    assert nb._empty((2,), None, like, Stream).dtype == nb._empty((2,), None, like, None).dtype
    assert nb._scratch(1000, like, None, Stream).numel() == nb._scratch(1000, like, None, None).numel() == 1000
    assert nb._scratch(0, like, None, Stream).numel() == 256 and nb._scratch(1000, like, like, Stream) is like


def test_arguments_that_are_none_are_refused():
    n, like = nb._native(), torch.zeros(1)
    for bad in ((None, like, torch.uint8, 1), (None, like, 5, 1, 3), (None, 5, torch.uint8, 1, 3), (None, like, torch.uint8, 1, 1.5),
                (None, like, torch.uint8, None, 3), (None, like, torch.uint8, 1, 1, 1, 1, 1, 1)):
        with pytest.raises(TypeError):
            n.empty_on(*bad)
    for bad in (lambda: n.empty_rows(like, 4, 8, None, None), lambda: n.empty_rows(like, 4), lambda: n.expert_buffers(like, 1, 1, 1, 128, None, None)):
        with pytest.raises(TypeError):
            bad()
    with pytest.raises(RuntimeError):
        n.empty_on(None, like, torch.uint8, 1, -1)
