"""The status calls work on the stream they are given: they neither wait for
the default stream nor leave anything on it."""
import pytest
import torch

from paper_2608_15797_gb300 import kvr
from tests.test_gpu_kv4 import dev, rnd

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    torch.cuda.set_device(0)


def busy_default_stream():
    """About 0.3 s of work on the default stream; the event behind it."""
    torch.cuda._sleep(600_000_000)
    e = torch.cuda.Event()
    e.record()
    return e


def test_kv4_status_on_a_stream_of_its_own():
    c = kvr.Kv4Cache(1, 1, 1, 7, 128, 5000)
    x = dev(rnd(1, (1, 1, 5000, 128)))
    c.load(0, x, x)
    q = dev(rnd(2, (1, 1, 1, 7, 128)))
    want = c.attend(q)
    view = c.scores_view()
    end = view.data_ptr() - c.buf.data_ptr() + 4 * view.stride(2)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    c.sync_status(st)  # what is loaded at first use is there
    with torch.cuda.stream(st):
        c.buf[end:c.nbytes] = 1
        ws, out = c.attend_workspace(1), torch.empty_like(want)
    st.synchronize()
    event = busy_default_stream()
    with pytest.raises(kvr.KvrError, match="KVR_EDEVICE"):
        c.sync_status(st)
    c.sync_status(st)
    assert not event.query()
    c.attend(q, out=out, workspace=ws, stream=st)
    st.synchronize()
    assert not event.query()
    assert torch.equal(out, want)


def test_cache_status_and_import_on_a_stream_of_their_own():
    """The evicted cache's status, with an error and without, and an import that
    a step on the same stream decodes from."""
    c = kvr.Cache(1, 1, 1, 2, 128, 40)
    x = dev(rnd(1, (1, 1, 20, 128)))
    c.load(0, x, x)
    step = [dev(rnd(2 + i, (1, 1, h, 128))) for i, h in enumerate((2, 1, 1))]
    state = c.export(0)
    want = c.step(*step, 16, 8)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    out = torch.empty_like(want)
    bad = torch.full_like(step[0], float("nan"))
    torch.cuda.synchronize()
    c.import_state(0, state, st)
    c.sync_status(st)
    event = busy_default_stream()
    c.step(bad, *step[1:], 16, 8, out=out, stream=st)
    with pytest.raises(kvr.KvrError, match="KVR_EDEVICE"):
        kvr.kvr_sync_status(c.handle, st)
    c.import_state(0, state, st)
    c.step(*step, 16, 8, out=out, stream=st)
    kvr.kvr_sync_status(c.handle, st)
    assert not event.query()
    assert torch.equal(out, want)


def test_detector_status_on_a_stream_of_its_own():
    det = kvr.EntropyDetector(2, 1000)
    logits = dev(rnd(1, (2, 1000)))
    bad = logits.clone()
    bad[1, 7] = float("nan")
    st = torch.cuda.Stream()
    outs = [torch.empty(2, dtype=t, device="cuda") for t in
            (torch.float32, torch.float32, torch.int32)]
    det.step(logits, *outs)
    torch.cuda.synchronize()
    det.sync_status(st)
    event = busy_default_stream()
    det.step(bad, *outs, stream=st)
    with pytest.raises(kvr.KvrError, match="KVR_EDEVICE"):
        det.sync_status(st)
    det.step(logits, *outs, stream=st)
    det.sync_status(st)
    assert not event.query()
