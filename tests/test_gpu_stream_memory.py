"""Memory that a call on a stream other than the current one allocates comes
from that stream's pool: a block that the current stream gave back, and may
still be working on, is not written by another."""
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


def given_back(nbytes, n=4):
    """Addresses of blocks of this size that the current stream has just given
    back: the next of that size on it would be one of them."""
    x = [torch.empty(nbytes, dtype=torch.uint8, device="cuda")
         for _ in range(n)]
    torch.cuda.synchronize()
    return {t.data_ptr() for t in x}


@pytest.mark.parametrize("raw", [False, True])
def test_outputs_and_scratch(raw):
    S, T, V = 2, 3, 1 << 20
    c = kvr.Kv4Cache(S, 1, 2, 7, 128, 600)
    for s in range(S):
        x = dev(rnd(s, (1, 2, 500, 128)))
        c.load(s, x, x)
    q = dev(rnd(3, (S, 1, T, 14, 128)))
    logits = dev(rnd(4, (S, T + 1, 1000)))
    tokens = torch.zeros((S, T), dtype=torch.int32, device="cuda")
    u, race = torch.zeros((S, T), device="cuda"), torch.ones(
        (S, 1000), device="cuda")
    st = torch.cuda.Stream()
    stream = st.cuda_stream if raw else st
    torch.cuda.synchronize()

    def check(call, nbytes):
        old = given_back(nbytes)
        assert torch.empty(nbytes, dtype=torch.uint8,
                           device="cuda").data_ptr() in old
        old = given_back(nbytes)
        got = call()
        st.synchronize()
        for t in got:
            assert t.data_ptr() not in old

    want = c.attend(q)
    out = []
    check(lambda: out.append(c.attend(q, stream=stream)) or out,
          want.nbytes)
    assert torch.equal(out[0], want)
    rows = c.read_newest(500)
    got = []
    check(lambda: got.extend(c.read_newest(500, stream=stream)) or got,
          rows[0].nbytes)
    assert all(map(torch.equal, got, rows))
    check(lambda: kvr.verify_drafts(logits, logits[:, :T].contiguous(), tokens,
                                    u, race, stream=stream), 4 * S)
    check(lambda: [kvr._scratch(V, "cuda", stream)], V)
    check(lambda: [kvr.Kv4Cache(S, 1, 2, 7, 128, 600, stream=stream).buf],
          c.nbytes)
