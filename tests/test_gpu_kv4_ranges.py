"""Attention over the 4-bit cache where values are tiny.  Bounds as in
test_gpu_kv4; a step below 2^-126 may count as 2^-126, which moves a value by
less than 15 * 2^-126."""
import numpy as np
import pytest
import torch

from oracle import kv4
from tests.test_gpu_kv4 import LOGIT, Pair, dev, rnd

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    torch.cuda.set_device(0)


@pytest.mark.parametrize("alone", [False, True])
@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("d,G,T", [(128, 2, 1), (64, 7, 1), (128, 3, 4),
                                   (64, 2, 5), (128, 7, 5)])
def test_steps_below_the_least_normal(d, G, T, out, alone):
    """Groups of V whose step is subnormal: zeros and one 1e-38, a spread of
    1.5e-37 around zero and above it; alone, or each beside ordinary rows."""
    n = 150
    v = rnd(2, (1, 1, n, 1, d))
    tiny = np.zeros((3, d), np.float32)
    tiny[0, 5::64] = 1e-38
    tiny[1] = 1e-38 * (np.arange(d) % 16) - 7e-38
    tiny[2] = 3e-37 + 1e-38 * (np.arange(d) % 13)
    rows = range(n) if alone else range(0, n, 7)
    for i in rows:
        v[0, 0, i, 0] = kv4.bf16(tiny[i % 3])
    s = kv4.quantise(v)[2]
    assert ((s > 0) & (s < 2.0**-126)).any()
    k = rnd(1, v.shape)
    q = rnd(4, (1, 1, T, G, d))
    p = Pair(1, 1, 1, G, d, n, "bf16", out)
    p.append(k, v)
    got = p.c.attend(dev(q)).float().cpu().numpy()[0, 0]
    ref, _, mag = kv4.attend(q[0, 0], kv4.values(k[0, 0, :, 0]),
                             kv4.values(v[0, 0, :, 0]))
    rel = 2.0**-8 if out == "bf16" else 2.0**-24
    half = 2.0**-11 if out == "bf16" else 0
    tol = rel * np.abs(ref) + mag * (LOGIT + half) + 15 * 2.0**-126 + 2.0**-122
    assert (np.abs(got - ref) <= tol).all()
    p.c.sync_status()
