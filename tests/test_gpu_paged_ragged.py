"""A batch whose sequences share a pool that one of them may fill: outputs on either
side of the sizes where the attention goes from a cluster a unit to spans of tiles,
with the pool dealt out evenly, held by the first, the last or a middle one."""
import pytest
import torch

from tests.test_gpu_paged import Book, dev, rnd

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    torch.cuda.set_device(0)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 64)])
@pytest.mark.parametrize("S,H,tiles", [
    (18, 1, 511), (18, 1, 512), (18, 1, 513), (9, 1, 1024), (9, 1, 1025),
    (4, 4, 512), (4, 4, 516), (2, 1, 1024), (2, 1, 1026)])
def test_one_sequence_holds_the_pool(dtype, d, S, H, tiles):
    b = Book(S, 1, H, 7, d, tiles, 16, tiles, dtype, "f32")
    k = rnd(tiles, (S, 1, 16 * tiles, H, d), dtype)
    v = k[..., ::-1]
    most = 16 * (tiles - S + 1)
    for lens in ([16 * (tiles // S) - 3] * S,
                 [most] + [1] * (S - 1), [16] * (S - 1) + [most - 5],
                 [0] * (S // 2) + [16 * tiles] + [0] * (S - S // 2 - 1)):
        b.plan([0] * S)
        n = max(lens)
        b.grow(lens, k=k[:, :, :n], v=v[:, :, :n])
        b.check_attend()
        q = b.queries()
        got = torch.empty((S, 1, H, tiles), dtype=torch.int32, device="cuda")
        out = b.c.attend_pages(dev(q, dtype), tiles - 1, 1, pages=got)
        b.check_out(q, out.cpu().numpy())
    b.c.sync_status()
