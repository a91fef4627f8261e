"""kvr_kv4_* and kvr_verify_* refuse bad arguments on the host, before any
device call."""
import ctypes

from paper_2608_15797_gb300 import kvr

lib = kvr.lib
ONE = ctypes.c_void_p(16)


def test_required_bytes():
    d = kvr.make_desc(2, 3, 4, 7, 128, 100)
    n = lib.kvr_kv4_required_bytes(ctypes.byref(d))
    rows = 2 * 3 * 4 * 100
    assert rows * (144 + 4) <= n < kvr.kvr_cache_required_bytes(d) / 2
    for bad in (kvr.make_desc(2, 3, 4, 9, 128, 100),
                kvr.make_desc(2, 3, 4, 7, 96, 100),
                kvr.make_desc(2, 3, 4, 7, 128, 0)):
        assert lib.kvr_kv4_required_bytes(ctypes.byref(bad)) == 0
    assert lib.kvr_kv4_required_bytes(None) == 0


def test_create_and_null_handles():
    d = kvr.make_desc(1, 1, 1, 1, 64, 8)
    need = lib.kvr_kv4_required_bytes(ctypes.byref(d))
    h = ctypes.c_void_p()
    for ptr, n, want in ((None, need, kvr.KVR_EINVAL),
                         (ctypes.c_void_p(0x1008), need, kvr.KVR_EINVAL),
                         (ctypes.c_void_p(0x1000), need - 1, kvr.KVR_ENOMEM)):
        assert lib.kvr_kv4_create(ctypes.byref(d), ptr, n, None,
                                  ctypes.byref(h)) == want and not h.value
    assert lib.kvr_kv4_create(ctypes.byref(d), ctypes.c_void_p(0x1000), need,
                              None, None) == kvr.KVR_EINVAL
    lib.kvr_kv4_destroy(None)
    E = kvr.KVR_EINVAL
    assert lib.kvr_kv4_load(None, 0, ONE, ONE, 1, None) == E
    assert lib.kvr_kv4_append(None, 0, 1, 1, None, ONE, ONE, None) == E
    assert lib.kvr_kv4_truncate(None, None) == E
    assert lib.kvr_kv4_lengths(None, None) == E
    assert lib.kvr_kv4_read(None, 0, 1, 1, None, ONE, ONE, None) == E
    assert lib.kvr_kv4_attend(None, 0, 1, 1, None, ONE, ONE, 0, ONE, 1, None) == E
    assert lib.kvr_kv4_attend_workspace_bytes(None, 0, 1, 1) == 0
    assert lib.kvr_kv4_evict(None, None, 1, 1, None) == E
    assert lib.kvr_kv4_scores(None, None, None) == E
    assert lib.kvr_kv4_launch_count(None, None) == E
    assert lib.kvr_kv4_sync_status(None, None) == E
    assert lib.kvr_cache_rows(None, None, None) == E


def _verify(d, target=ONE, ts=None, tokens=ONE, ws=ONE, n=1 << 30):
    return lib.kvr_verify_drafts(
        ctypes.byref(d) if d else None, target, ts or 100, ONE, 100, tokens,
        ONE, ONE, None, ONE, ONE, ws, n, None)


def test_verify_arguments():
    good = kvr.kvr_verify_desc(2, 3, 100, 1.0, kvr.KVR_BF16)
    assert lib.kvr_verify_workspace_bytes(ctypes.byref(good)) > 0
    for bad in ((0, 3, 100, 1.0, 0), (70000, 3, 100, 1.0, 0),
                (2, -1, 100, 1.0, 0), (2, 65, 100, 1.0, 0), (2, 3, 0, 1.0, 0),
                (2, 3, 100, -1.0, 0), (2, 3, 100, float("nan"), 0),
                (2, 3, 100, float("inf"), 0), (2, 3, 100, 1.0, 7)):
        d = kvr.kvr_verify_desc(*bad)
        assert lib.kvr_verify_workspace_bytes(ctypes.byref(d)) == 0
        assert _verify(d) == kvr.KVR_EINVAL
    assert _verify(None) == kvr.KVR_EINVAL
    assert _verify(good, target=None) == kvr.KVR_EINVAL
    assert _verify(good, tokens=None) == kvr.KVR_EINVAL
    assert _verify(good, ts=99) == kvr.KVR_EINVAL
    assert _verify(good, ws=None) == kvr.KVR_EINVAL
    assert _verify(good, ws=ctypes.c_void_p(8)) == kvr.KVR_EINVAL
    assert _verify(good, n=0) == kvr.KVR_ENOMEM
