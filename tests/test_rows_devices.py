"""Which device and stream the calls on dense rows go to (CPU only: devices are stood in for)."""
import types

import pytest
import torch

from paper_2102_05187_amd import binding


@pytest.fixture
def current(monkeypatch):
    """Two devices, the first one current; what is entered is noted."""
    now = [0]

    class Device:
        def __init__(self, device):
            self.index = torch.device(device).index

        def __enter__(self):
            self.before, now[0] = now[0], self.index

        def __exit__(self, *_):
            now[0] = self.before

    monkeypatch.setattr(binding, "_raw_device", lambda: now[0])
    monkeypatch.setattr(binding, "_raw_stream", lambda index: 1000 + index)
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: True)
    monkeypatch.setattr(torch.cuda, "device", Device)
    return now


def launch(current, monkeypatch, device, stream=None):
    seen = []

    def comet_anything(*args):
        seen.append((current[0], *args))
        return 0

    monkeypatch.setattr(binding, "_lib", lambda: types.SimpleNamespace(comet_anything=comet_anything))
    try:
        binding._call("comet_anything", torch.device(device), stream, 5)
    finally:
        assert current[0] == 0
    return seen


def test_the_operands_device_is_made_current(current, monkeypatch):
    assert launch(current, monkeypatch, "cuda:0") == [(0, 5, 1000)]
    assert launch(current, monkeypatch, "cuda:1") == [(1, 5, 1001)]


def test_a_stream_goes_with_its_device(current, monkeypatch):
    stream = types.SimpleNamespace(device=torch.device("cuda:1"), cuda_stream=77)
    assert launch(current, monkeypatch, "cuda:1", stream) == [(1, 5, 77)]
    with pytest.raises(ValueError):
        launch(current, monkeypatch, "cuda:0", stream)
