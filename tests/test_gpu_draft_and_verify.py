"""The example that runs the 4-bit cache, its cut and the verification
together: what it emits is what the model over the full cache emits."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    torch.cuda.set_device(0)


def prompts(m, lens):
    g = torch.Generator().manual_seed(5)
    return [torch.randint(m.V, (n,), generator=g).tolist() for n in lens]


@pytest.mark.parametrize("draft,budget,window", [(1, 8, 4), (4, 32, 8),
                                                 (6, 400, 16)])
def test_cold_draws_are_the_greedy_tokens(draft, budget, window):
    """At a temperature near zero the target's softmax has one token, so every
    round emits what greedy decoding over the full cache does, whatever was
    drafted from however few rows."""
    from examples import draft_and_verify as ex
    m = ex.Decoder(seed=7)
    p = prompts(m, (150, 1, 77))
    out, share = ex.generate(m, p, 24, draft, budget, window, 1e-5)
    want = ex.greedy(m, p, 24)
    for got, ref in zip(out, want):
        assert got[:24] == ref
    assert 0 <= share <= 1


def test_command(capsys):
    from examples import draft_and_verify as ex
    ex.main(["--seqs", "2", "--prompt", "60", "--new", "12"])
    text = capsys.readouterr().out
    assert "sequence 1: 23 + " in text and "accepted" in text
