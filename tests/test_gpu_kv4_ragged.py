"""What lies in a ragged call's padding, the tokens from counts[s] on, does not
matter to the 4-bit cache's attention: outputs and accumulated weights are bit
for bit those of a call whose padding is zeros."""
import numpy as np
import pytest
import torch

from tests.test_gpu_kv4 import Pair, dev, rnd

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    torch.cuda.set_device(0)


@pytest.mark.parametrize("fill", [np.nan, np.inf, -3e38])
@pytest.mark.parametrize("dtype,out,d,G,T", [
    ("bf16", "bf16", 128, 7, 3), ("bf16", "bf16", 64, 7, 3),
    ("f32", "f32", 128, 7, 3), ("f32", "f32", 64, 5, 9),
    ("bf16", "f32", 128, 3, 4), ("bf16", "bf16", 64, 7, 12),
    ("bf16", "bf16", 128, 7, 5), ("bf16", "bf16", 128, 8, 40),
])
def test_padding_of_a_ragged_call(dtype, out, d, G, T, fill):
    lens = [200, 130, 90, 65, 400]
    counts = [T, 1, 0, 2, T - 1]
    p = Pair(5, 1, 2, G, d, 400, dtype, out)
    for s, n in enumerate(lens):
        p.load(s, n, 20 + s)
    q = rnd(3, (5, 1, T, 2 * G, d), dtype)
    got = []
    for pad in (0.0, fill):
        p.c.scores_view().zero_()
        for s, m in enumerate(counts):
            q[s, :, m:] = pad
        o = p.c.attend(dev(q, dtype), counts=counts, scores=True)
        got.append((o.float().cpu().numpy(), p.c.scores_view().cpu().numpy()))
    for a, b in zip(*got):
        np.testing.assert_array_equal(a, b)
    assert np.isfinite(got[1][1]).all()
    p.c.sync_status()
