"""The binding of the 4-bit cache and of the verification refuses, before the
library is called, tensors that do not lie on the GPU, workspaces with gaps, and
a destination of the wrong kind."""
import pytest
import torch

from paper_2608_15797_gb300 import kvr


@pytest.fixture
def cache(monkeypatch):
    """A Kv4Cache of cuda:0 without its handle."""
    class Forbidden:
        def __getattr__(self, name):
            if name == "kvr_kv4_attend_workspace_bytes":
                return lambda *a: 1024

            def called(*a):
                raise AssertionError(f"{name} was called")
            return called
    c = kvr.Kv4Cache.__new__(kvr.Kv4Cache)
    c.S, c.L, c.H, c.G, c.d, c.cap = 2, 1, 1, 2, 128, 64
    c.dtype = c.out_dtype = "bf16"
    c._io = c._out = torch.bfloat16
    c._all, c._scores, c._device, c.handle = (0, 1), None, 0, None
    c.buf = torch.zeros(16, dtype=torch.uint8)
    monkeypatch.setattr(kvr, "lib", Forbidden())
    return c


def host(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype)


def test_tensors_of_the_host_are_refused(cache):
    rows = host(2, 1, 3, 1, 128)
    for call in (lambda: cache.load(0, host(1, 1, 3, 128), host(1, 1, 3, 128)),
                 lambda: cache.append(rows, rows),
                 lambda: cache.attend(host(2, 1, 3, 2, 128))):
        with pytest.raises(ValueError, match="must lie on the GPU"):
            call()


class Elsewhere:
    """What the binding asks of a tensor, of one on another GPU."""

    def __init__(self, t, device):
        self.t, self.at = t, device

    def get_device(self):
        return self.at

    def __getattr__(self, name):
        return getattr(self.t, name)


def test_out_and_workspace_lie_with_the_cache(cache):
    q = Elsewhere(host(2, 1, 3, 2, 128), 0)
    for at in (-1, 1):
        out = Elsewhere(host(2, 1, 3, 2, 128), at)
        with pytest.raises(ValueError, match="out must lie on the GPU"):
            cache.attend(q, out=out)
        ws = Elsewhere(host(4096, dtype=torch.uint8), at)
        with pytest.raises(ValueError, match="workspace must lie on the GPU"):
            cache.attend(q, out=Elsewhere(out.t, 0), workspace=ws)
    gaps = Elsewhere(host(1, dtype=torch.uint8).expand(4096), 0)
    with pytest.raises(ValueError, match="contiguous"):
        cache.attend(q, out=Elsewhere(out.t, 0), workspace=gaps)


def test_the_destination_of_a_cut(cache):
    with pytest.raises(ValueError, match="must be a Cache"):
        cache.evict_into(cache, 4, 4)
    other = kvr.Cache.__new__(kvr.Cache)
    other.buf, other.handle = host(16, dtype=torch.uint8), None
    with pytest.raises(ValueError, match="destination must lie on the GPU"):
        cache.evict_into(other, 4, 4)


def test_a_buffer_of_the_host():
    n = 1 << 20
    with pytest.raises(ValueError, match="buf must lie on the GPU"):
        kvr.Kv4Cache(1, 1, 1, 1, 64, 8, buf=torch.zeros(n, dtype=torch.uint8))


def test_verification():
    S, T, V = 2, 3, 50
    x = [host(S, T + 1, V), host(S, T, V), host(S, T, dtype=torch.int32),
         host(S, T, dtype=torch.float32), host(S, V, dtype=torch.float32)]
    with pytest.raises(ValueError, match="target must lie on the GPU"):
        kvr.verify_drafts(*x)
    names = ("draft", "tokens", "u", "race")
    for i, name in enumerate(names, 1):
        for at in (-1, 1):
            y = [Elsewhere(t, at if j == i else 0) for j, t in enumerate(x)]
            with pytest.raises(ValueError, match=f"{name} must lie on the GPU"):
                kvr.verify_drafts(*y)
