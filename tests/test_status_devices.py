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


@pytest.mark.parametrize("kind", [kvr.PagedCache, kvr.Kv4Cache])
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


def test_calls_of_the_4_bit_cache(current):
    """Its kernels would run on the current device, with the memory of another."""
    c = bare(kvr.Kv4Cache, 0)
    c.S, c.L, c.H, c.G, c.d = 2, 1, 1, 2, 128
    c.dtype = c.out_dtype = "bf16"
    c._io = c._out = torch.bfloat16
    c._all, c.buf = (0, 1), torch.zeros(16, dtype=torch.uint8)

    class Here:
        """What the binding asks of a tensor, of one on cuda:0."""

        def __init__(self, *shape, dtype=torch.bfloat16):
            self.t = torch.zeros(shape, dtype=dtype)

        def get_device(self):
            return 0

        def __getattr__(self, name):
            return getattr(self.t, name)

    rows, q = Here(2, 1, 3, 1, 128), Here(2, 1, 3, 2, 128)
    seq, ws = Here(1, 1, 3, 128), Here(4096, dtype=torch.uint8)
    other = kvr.Cache.__new__(kvr.Cache)
    other.buf, other.handle = Here(16, dtype=torch.uint8), None
    for call in (lambda: c.load(0, seq, seq), lambda: c.append(rows, rows),
                 lambda: c.read_newest(3),
                 lambda: c.attend(q, out=q, workspace=ws),
                 lambda: c.evict_into(other, 4, 4)):
        current[0] = 0
        with pytest.raises(Called) as e:
            call()
        assert e.value.args[1][-1] == 1000
        current[0] = 1
        with pytest.raises(ValueError, match="current device"):
            call()
