"""Which stream a call of the binding goes to.  The default stream's handle is 0 on every device, and a launch there goes to the current one:
a detector of another device refuses it.  Streams that have handles know their device.  No GPU is needed."""
from types import SimpleNamespace

import pytest
import torch

from paper_2605_17879_amd.guard import Detector, GuardError


def detector(index, current, handle=0):
    """What Detector._stream takes of a detector."""
    return SimpleNamespace(device=torch.device("cuda") if index is None else torch.device("cuda", index), _index=index, _torch=torch,
                           _raw_stream=lambda i: handle, _current=lambda: current)


@pytest.mark.parametrize("stream", [None, SimpleNamespace(cuda_stream=0)])
def test_the_default_stream_of_another_device_is_refused(stream):
    with pytest.raises(GuardError, match="cuda:1"):
        Detector._stream(detector(1, 0), stream)
    assert Detector._stream(detector(1, 1), stream) == 0


def test_streams_that_have_a_handle_are_taken():
    assert Detector._stream(detector(1, 0, handle=77), None) == 77
    assert Detector._stream(detector(1, 0), SimpleNamespace(cuda_stream=99)) == 99


def test_a_detector_of_whichever_device_is_current():
    assert Detector._stream(detector(None, 3), SimpleNamespace(cuda_stream=0)) == 0
