"""The tensors of a call to the operators around the attention lie on the
current device (CPU, with stand-ins for tensors)."""
import pytest


class On:
    def __init__(self, device):
        self.index = device

    def get_device(self):  # -1: host memory
        return self.index


@pytest.fixture
def fv(monkeypatch):
    from paper_2609_36757_gb300 import build
    build.build()
    from paper_2609_36757_gb300 import fastvr
    fastvr._setup()
    monkeypatch.setattr(fastvr, "_current_device", lambda: 1)
    monkeypatch.setattr(fastvr, "_raw_stream", lambda i: 100 + i)
    return fastvr


def test_stream_of_the_current_device(fv):
    assert fv._stream_of(On(1)) == 101
    assert fv._stream_of(On(1), None, On(1)) == 101


@pytest.mark.parametrize("devices", [(0,), (-1,), (0, 0), (1, 0), (1, -1),
                                     (1, 1, 0), (1, 1, -1), (0, 1)])
def test_other_places_are_refused(fv, devices):
    with pytest.raises(ValueError):
        fv._stream_of(*map(On, devices))
    with pytest.raises(ValueError):
        fv._stream_of(On(devices[0]), None, *map(On, devices[1:]))
