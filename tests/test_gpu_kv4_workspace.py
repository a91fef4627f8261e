"""kvr_kv4_attend_workspace_bytes: what serves a call of n tokens serves every
call of fewer."""
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


@pytest.mark.parametrize("S,H,G,d,cap,dtype", [
    (4, 4, 7, 128, 4096, "bf16"), (2, 2, 1, 128, 1000, "bf16"),
    (3, 2, 5, 64, 700, "bf16"), (2, 1, 8, 128, 5000, "f32")])
def test_more_tokens_need_no_less(S, H, G, d, cap, dtype):
    c = kvr.Kv4Cache(S, 1, H, G, d, cap, dtype=dtype, out_dtype=dtype)
    need = [int(kvr.lib.kvr_kv4_attend_workspace_bytes(c.handle, 0, 1, n))
            for n in range(1, 1400)]
    assert need == sorted(need)
    assert c.attend_workspace(147).numel() == need[146]


def test_one_workspace_serves_fewer_tokens():
    c = kvr.Kv4Cache(4, 1, 2, 7, 128, 4096)
    for s in range(4):
        x = dev(rnd(s, (1, 2, 4000, 128)))
        c.load(s, x, x)
    most = int(kvr.lib.kvr_kv4_attend_workspace_bytes(c.handle, 0, 1, 4))
    ws = torch.empty(most, dtype=torch.uint8, device="cuda")
    for n in (1, 2, 3, 4):
        q = dev(rnd(n, (4, 1, n, 14, 128)))
        out = c.attend(q, workspace=ws)
        assert torch.equal(out, c.attend(q))
    with pytest.raises(kvr.KvrError, match="KVR_ENOMEM"):
        c.attend(q, workspace=ws[:16])
    c.sync_status()
