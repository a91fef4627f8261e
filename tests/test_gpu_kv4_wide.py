"""Attention over the 4-bit cache where it is wide or far: many query rows a
unit, units cut over many blocks, references that are outgrown, rows that few
tokens see, and offsets past 32 bits.  Bounds as in test_gpu_kv4."""
import numpy as np
import pytest
import torch

from oracle import kv4
from paper_2608_15797_gb300 import kvr
from tests.test_gpu_kv4 import Pair, dev, rnd

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    torch.cuda.set_device(0)


@pytest.mark.parametrize("d,G,T,n", [
    (128, 7, 160, 200),   # more column tiles than are cut over blocks
    (128, 1, 1100, 1100),  # the same, a whole prompt at once
    (64, 7, 64, 150),
    (128, 5, 5, 129),     # 25 rows: the least for tensor memory
    (128, 3, 8, 129),     # 24: the most for the other kernel
    (128, 5, 13, 300),    # 65: one row more than a tile
    (128, 3, 87, 300),    # 261: a second pass of the scores
])
def test_many_query_rows(d, G, T, n):
    p = Pair(1, 1, 2, G, d, n)
    p.load(0, n, 3)
    p.check_attend(rnd(5, (1, 1, T, 2 * G, d)), scores=True)


@pytest.mark.parametrize("T,n", [(5, 5000), (32, 5000), (5, 513), (5, 512)])
def test_one_unit_over_the_whole_gpu(T, n):
    p = Pair(1, 1, 1, 7, 128, n)
    p.load(0, n, 11)
    p.check_attend(rnd(6, (1, 1, T, 7, 128)), scores=True)


def test_many_sequences_wide():
    lens = [1 + (37 * s) % 300 for s in range(131)]
    counts = [min(n, s % 5) for s, n in enumerate(lens)]
    p = Pair(131, 1, 1, 7, 128, 300)
    for s, n in enumerate(lens):
        p.load(s, n, s)
    p.check_attend(rnd(7, (131, 1, 4, 7, 128)), counts=counts, scores=True)


@pytest.mark.parametrize("T", [1, 5, 13])
def test_references_that_are_outgrown(T):
    """Logits that grow along the context, to about 25: every tile's largest
    is far above the one before."""
    n, G = 1500, 7
    p = Pair(1, 1, 1, G, 128, n)
    u = rnd(1, (1, 1, 1, 128))
    k = kv4.bf16(u * np.linspace(0, 2.2, n, dtype=np.float32)[:, None])
    v = rnd(2, (1, 1, n, 128))
    p.c.load(0, dev(k), dev(v))
    p.k[0], p.v[0] = k, v
    q = kv4.bf16(np.broadcast_to(u[0, 0], (1, 1, T, G, 128)) *
                 np.linspace(-0.5, 1, T * G, dtype=np.float32).reshape(
                     1, 1, T, G, 1))
    p.check_attend(q, scores=True)


def test_non_finite_rows_wide():
    """26 query rows: a NaN key or value in the newest row but one reaches the
    last two tokens, one of a value only its 64 channels."""
    T, G = 13, 2
    p = Pair(2, 1, 1, G, 128, 400)
    for s in range(2):
        p.load(s, 250 + 60 * s, 3 + s)
    k, v = (rnd(i, (2, 1, T, 1, 128)) for i in (4, 5))
    k[0, 0, T - 2, 0, 5] = np.nan
    v[1, 0, T - 2, 0, 70] = np.inf
    p.append(k, v)
    q = rnd(2, (2, 1, T, G, 128))
    got = p.c.attend(dev(q)).float().cpu().numpy()
    assert np.isnan(got[0, 0, T - 2:]).all()
    assert np.isnan(got[1, 0, T - 2:, :, 64:]).all()
    for s in range(2):
        n = p.k[s].shape[2] - T
        for t in range(T):
            kk = kv4.values(p.k[s][0, 0, :n + t + 1])
            vv = kv4.values(p.v[s][0, 0, :n + t + 1])
            if t >= T - 2:
                if s == 0:
                    continue
                vv[:, 64:] = 0
            want, _, _ = kv4.attend(q[s, 0, t:t + 1], kk, vv)
            d = 64 if t >= T - 2 else 128
            np.testing.assert_allclose(got[s, 0, t, :, :d], want[0, :, :d],
                                       atol=2e-2)
    with pytest.raises(kvr.KvrError):
        p.c.sync_status()


@pytest.mark.parametrize("T,G", [(1, 6), (5, 7)])
def test_units_past_32_bits(T, G):
    """The last of sequences whose units lie 2^32 bytes and more into the
    buffer: 16 of 2^21 rows."""
    p = Pair(16, 1, 1, G, 128, 1 << 21)
    for s in (0, 15):
        p.load(s, 300 + s, s)
    for s in range(1, 15):
        p.load(s, T, s)
    p.check_attend(rnd(3, (16, 1, T, G, 128)), scores=True)
    k, _ = p.c.read_newest(1)
    for s in (0, 15):
        np.testing.assert_array_equal(
            k[s, 0, 0, 0].float().cpu().numpy(),
            kv4.bf16(kv4.values(p.k[s][0, 0, -1:])[0]))


@pytest.mark.parametrize("T,G", [(1, 1), (5, 7)])
def test_rows_past_31_bits(T, G):
    """A unit of nearly 2^24 rows, 2.4 GB: only the tokens at its end matter,
    as every other key gives a logit of 0 and theirs 181."""
    n = (1 << 24) - T
    c = kvr.Kv4Cache(1, 1, 1, G, 128, 1 << 24)
    x = torch.zeros((1, 1, n, 128), dtype=torch.bfloat16, device="cuda")
    c.load(0, x, x)
    del x
    four = torch.full((1, 1, T, 1, 128), 4.0, dtype=torch.bfloat16,
                      device="cuda")
    v = rnd(1, (1, 1, T, 1, 128))
    c.append(four, dev(v))
    out = c.attend(four.expand(1, 1, T, G, 128).contiguous(), scores=True)
    val = kv4.values(v[0, 0, :, 0]).astype(np.float64)
    got = out.float().cpu().numpy()[0, 0]
    for t in range(T):
        want = val[:t + 1].mean(0)
        tol = 2.0**-8 * np.abs(want) + np.abs(val[:t + 1]).mean(0) * (
            2e-5 + 2.0**-11)
        assert (np.abs(got[t] - want) <= tol).all()
    score = c.scores_view()[0, 0, 0]
    assert float(score[:n].abs().max()) < 1e-9
    want = [sum(1 / (t + 1) for t in range(j, T)) for j in range(T)]
    np.testing.assert_allclose(score[n:n + T].cpu().numpy(), want, rtol=1e-4)
    c.sync_status()


@pytest.mark.parametrize("T", [1, 5])
def test_status_clears_what_a_launch_that_gave_up_left(T):
    """Behind the scores lie the arrivals of units that CTAs share and the
    error word; with the error reported all of them are cleared, and units that
    are cut are joined rightly again."""
    p = Pair(1, 1, 1, 7, 128, 5000)
    p.load(0, 5000, 11)
    view = p.c.scores_view()
    end = view.data_ptr() - p.c.buf.data_ptr() + 4 * view.stride(2)
    p.c.buf[end:p.c.nbytes] = 1
    with pytest.raises(kvr.KvrError, match="KVR_EDEVICE"):
        p.c.sync_status()
    p.check_attend(rnd(6, (1, 1, T, 7, 128)), scores=True)
    p.c.sync_status()
