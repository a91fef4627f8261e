"""kvr_paged_* refuse bad arguments on the host, before any device call."""
import ctypes

import pytest
import torch

from paper_2608_15797_gb300 import kvr

lib = kvr.lib
ONE = ctypes.c_void_p(16)
GOOD = dict(n_seq=2, n_layers=3, n_kv_heads=4, group=7, head_dim=128,
            n_pages=10, page_rows=64, table_pages=5)


def desc(**kw):
    return kvr.PagedCache.make_desc(**{**GOOD, **kw})


def test_required_bytes():
    n = kvr.PagedCache.required_bytes(**GOOD)
    rows = 3 * 4 * 10 * 64 * 128 * 2
    assert 2 * rows + rows // 32 <= n < 2 * rows + rows // 32 + 20000
    assert kvr.PagedCache.required_bytes(**{**GOOD, "dtype": "f32"}) > 2 * n - 40000
    for bad in (dict(n_seq=0), dict(n_seq=65536), dict(n_layers=0),
                dict(n_kv_heads=0), dict(group=0), dict(group=9),
                dict(head_dim=96), dict(n_pages=0), dict(table_pages=0),
                dict(page_rows=8), dict(page_rows=48), dict(page_rows=256),
                dict(n_pages=1 << 25), dict(table_pages=1 << 25),
                dict(n_layers=65535, n_kv_heads=2),
                dict(n_seq=65535, n_layers=32768),
                dict(n_layers=80, n_kv_heads=8, n_pages=840000),
                dict(softmax_scale=-1.0), dict(softmax_scale=float("nan")),
                dict(softmax_scale=float("inf"))):
        d = desc(**bad)
        assert lib.kvr_paged_required_bytes(ctypes.byref(d)) == 0, bad
    for field in ("kv_dtype", "out_dtype"):
        d = desc()
        setattr(d, field, 2)
        assert lib.kvr_paged_required_bytes(ctypes.byref(d)) == 0
    assert lib.kvr_paged_required_bytes(None) == 0
    # the largest pool: byte counts pass 32 bits
    big = desc(n_pages=800000, n_layers=80, n_kv_heads=8)
    assert lib.kvr_paged_required_bytes(ctypes.byref(big)) > \
        2 * 80 * 8 * 800000 * 64 * 256


def test_create_and_null_handles():
    d = desc()
    need = lib.kvr_paged_required_bytes(ctypes.byref(d))
    h = ctypes.c_void_p()
    for ptr, n, want in ((None, need, kvr.KVR_EINVAL),
                         (ctypes.c_void_p(0x1008), need, kvr.KVR_EINVAL),
                         (ctypes.c_void_p(0x1000), need - 1, kvr.KVR_ENOMEM)):
        assert lib.kvr_paged_create(ctypes.byref(d), ptr, n, None,
                                    ctypes.byref(h)) == want and not h.value
    assert lib.kvr_paged_create(ctypes.byref(d), ctypes.c_void_p(0x1000), need,
                                None, None) == kvr.KVR_EINVAL
    assert lib.kvr_paged_create(None, ctypes.c_void_p(0x1000), need, None,
                                ctypes.byref(h)) == kvr.KVR_EINVAL
    lib.kvr_paged_destroy(None)
    E = kvr.KVR_EINVAL
    assert lib.kvr_paged_plan(None, ONE, 1, ONE, None) == E
    assert lib.kvr_paged_append(None, 0, 1, 1, 1, ONE, ONE, ONE, None) == E
    assert lib.kvr_paged_attend_workspace_bytes(None, 0, 1) == 0
    assert lib.kvr_paged_attend(None, 0, 1, ONE, ONE, ONE, 1 << 30, None) == E
    assert lib.kvr_paged_attend_pages_workspace_bytes(None, 0, 1, 1, 1) == 0
    assert lib.kvr_paged_attend_pages(None, 0, 1, ONE, 1, 1, ONE, None, ONE,
                                      1 << 30, None) == E
    assert lib.kvr_paged_tables(None, None, None, None, None) == E
    assert lib.kvr_paged_rows(None, None, None, None) == E
    assert lib.kvr_paged_launch_count(None, None) == E
    assert lib.kvr_paged_sync_status(None, None) == E
    assert "null" in kvr.kvr_last_error()


@pytest.fixture
def cache(monkeypatch):
    """A PagedCache of cuda:0 without its handle; no call may reach the
    library."""
    class Forbidden:
        def __getattr__(self, name):
            def called(*a):
                raise AssertionError(f"{name} was called")
            return called
    c = kvr.PagedCache.__new__(kvr.PagedCache)
    c.S, c.L, c.H, c.G, c.d = 2, 1, 1, 2, 128
    c._hg, c.n_pages, c.page_rows, c.table_pages = 2, 4, 16, 2
    c.dtype = c.out_dtype = "bf16"
    c._io = c._out = torch.bfloat16
    c._all, c._tables, c._pool = (0, 1), None, None
    c._device, c.handle = 0, None
    c.buf = torch.zeros(16, dtype=torch.uint8)
    monkeypatch.setattr(kvr, "lib", Forbidden())
    monkeypatch.setattr(kvr, "_raw_device", lambda: 0)
    monkeypatch.setattr(kvr, "_raw_stream", lambda device: 0)
    return c


def host(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype)


def i32(*shape):
    return host(*shape, dtype=torch.int32)


class Elsewhere:
    """What the binding asks of a tensor, of one on a GPU."""

    def __init__(self, t, device=0):
        self.t, self.at = t, device

    def get_device(self):
        return self.at

    def __getattr__(self, name):
        return getattr(self.t, name)


def test_tensors_of_another_memory_are_refused(cache):
    here = Elsewhere
    rows = host(2, 1, 3, 1, 128)
    q = host(2, 1, 2, 128)
    for at in (-1, 1):
        def there(t):
            return Elsewhere(t, at)
        for call in (
                lambda: cache.plan(there(i32(2))),
                lambda: cache.plan(here(i32(2)), 3, slots=there(i32(2, 3))),
                lambda: cache.append(here(rows), here(rows), there(i32(2, 3))),
                lambda: cache.append(there(rows), here(rows), here(i32(2, 3))),
                lambda: cache.append(here(rows), there(rows), here(i32(2, 3))),
                lambda: cache.attend(there(q)),
                lambda: cache.attend(here(q), out=there(q)),
                lambda: cache.attend(here(q), out=here(q), workspace=there(
                    host(99, dtype=torch.uint8))),
                lambda: cache.attend_pages(there(q), 1),
                lambda: cache.attend_pages(here(q), 1, out=here(q),
                                           pages=there(i32(2, 1, 1, 2))),
                lambda: cache.attend_pages(
                    here(q), 1, out=here(q),
                    workspace=there(host(99, dtype=torch.uint8)))):
            with pytest.raises(ValueError, match="must lie on the GPU"):
                call()


def test_shapes_types_and_gaps_are_refused(cache):
    h = Elsewhere
    rows, q = host(2, 1, 3, 1, 128), host(2, 1, 2, 128)
    gaps = host(2, 1, 4, 128)[:, :, ::2]
    for call in (lambda: cache.plan(h(i32(3))),
                 lambda: cache.plan(h(host(2))),
                 lambda: cache.plan(h(i32(2)), 3, slots=h(i32(2, 4))),
                 lambda: cache.append(h(rows), h(rows), h(i32(2, 4))),
                 lambda: cache.append(h(rows), h(rows), h(host(2, 3))),
                 lambda: cache.append(h(rows), h(rows.float()), h(i32(2, 3))),
                 lambda: cache.attend(h(q.float())),
                 lambda: cache.attend(h(gaps)),
                 lambda: cache.attend(h(q), out=h(q.float())),
                 lambda: cache.attend_pages(h(q), 1, out=h(q),
                                            pages=h(i32(2, 1, 1, 3)))):
        with pytest.raises(ValueError, match="must be contiguous"):
            call()
    for n in (-1, (1 << 24) + 1):
        with pytest.raises(ValueError, match="new tokens"):
            cache.plan(h(i32(2)), n)


def test_another_current_device_is_refused(cache, monkeypatch):
    monkeypatch.setattr(kvr, "_raw_device", lambda: 1)
    q = Elsewhere(host(2, 1, 2, 128))
    for call in (lambda: cache.plan(Elsewhere(i32(2))),
                 lambda: cache.attend(q), lambda: cache.attend_pages(q, 1)):
        with pytest.raises(ValueError, match="current device"):
            call()


def test_a_buffer_of_the_host():
    n = kvr.PagedCache.required_bytes(**GOOD)
    with pytest.raises(ValueError, match="buf must lie on the GPU"):
        kvr.PagedCache(**GOOD, buf=torch.zeros(n, dtype=torch.uint8))
    with pytest.raises(ValueError, match="at least"):
        kvr.PagedCache(**GOOD, buf=torch.zeros(n - 1, dtype=torch.uint8))
