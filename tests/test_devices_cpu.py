"""The binding's choice of a stream where the current device is not the tensors' (no GPU needed)."""
import pytest
import torch

import paper_2609_33390_amd as brisk


class Stream:
    def __init__(self, handle):
        self.cuda_stream = handle


@pytest.fixture
def current(monkeypatch):
    """Two devices: which is current, and each one's current stream."""
    now = {"device": 0, "streams": {0: 0, 1: 0}}
    monkeypatch.setattr(brisk, "_several_devices", True)
    monkeypatch.setattr(brisk, "_current_device", lambda: now["device"])
    monkeypatch.setattr(brisk, "_raw_stream", lambda index: now["streams"][index])
    return now


def test_a_default_stream_is_the_current_devices(current):
    one = torch.device("cuda", 1)
    assert brisk._stream_ptr(torch.device("cuda", 0), None) == 0
    for stream in (None, 0, Stream(0)):
        with pytest.raises(ValueError, match="cuda:1"):
            brisk._stream_ptr(one, stream)
    current["device"] = 1
    assert brisk._stream_ptr(one, None) == 0 and brisk._stream_ptr(one, 0) == 0


def test_other_streams_name_their_device(current):
    one = torch.device("cuda", 1)
    current["streams"][1] = 77
    assert brisk._stream_ptr(one, None) == 77
    assert brisk._stream_ptr(one, Stream(5)) == 5 and brisk._stream_ptr(one, 9) == 9


def test_host_devices_have_no_number_to_compare(current):
    assert brisk._stream_ptr(torch.device("cpu", 0), None) == 0
