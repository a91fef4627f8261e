"""The status of a cache is read on a stream of the cache's device: with another
device current the binding refuses the call, since it would wait for that device's
stream and could miss an error of kernels still running."""
import pytest
import torch

from paper_2608_15797_gb300 import kvr


class Called(Exception):
    pass


@pytest.fixture
def current(monkeypatch):
    """Which device is current, in current[0]; library calls raise Called."""
    class Library:
        def __getattr__(self, name):
            def called(*a):
                raise Called(name, a)
            return called
    at = [0]
    monkeypatch.setattr(kvr, "lib", Library())
    monkeypatch.setattr(kvr, "_raw_device", lambda: at[0])
    monkeypatch.setattr(kvr, "_raw_stream", lambda device: 1000 + device)
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: True)
    return at


def bare(kind, device):
    """A cache of this device without its handle."""
    c = kind.__new__(kind)
    c._device, c.handle = device, None
    return c


@pytest.mark.parametrize("kind", [kvr.PagedCache])
@pytest.mark.parametrize("device", [0, 1])
def test_status_on_the_caches_device(current, kind, device):
    c = bare(kind, device)
    current[0] = device
    with pytest.raises(Called) as e:
        c.sync_status()
    assert e.value.args[1] == (None, 1000 + device)
    with pytest.raises(Called) as e:
        c.sync_status(stream=77)
    assert e.value.args[1] == (None, 77)
    current[0] = 1 - device
    for stream in (None, 0, 77):
        with pytest.raises(ValueError, match="current device"):
            c.sync_status(stream)
