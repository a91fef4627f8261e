"""verify_drafts takes rows of logits that lie a stride apart, and refuses, on
the host, rows that overlap: the kernels read every row whole."""
import pytest
import torch

from paper_2608_15797_gb300 import kvr


@pytest.mark.parametrize("S,n", [(1, 4), (3, 1), (3, 4), (8, 2)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_overlapping_rows_are_refused(S, n, dtype):
    V = 100
    one = torch.zeros(1, 1, V, dtype=dtype)
    row = torch.zeros(V + S * n, dtype=dtype)
    for x in (one.expand(S, n, V), row.as_strided((S, n, V), (n, 1, 1)),
              row.as_strided((S, n, V), (0, 0, 1)),
              torch.zeros(S * n * V, dtype=dtype).as_strided(
                  (S, n, V), (n * (V - 1), V - 1, 1))):
        with pytest.raises(ValueError):
            kvr._logit_rows(x, "draft")


def test_rows_of_one_distribution_expanded_over_a_batch():
    """Expanded along one axis only, and whole calls with such logits."""
    S, T, V = 4, 3, 50
    x = torch.zeros(S, T + 1, V)
    for d in (torch.zeros(1, T, V).expand(S, T, V),
              torch.zeros(S, 1, V).expand(S, T, V),
              torch.zeros(V).expand(S, T, V)):
        with pytest.raises(ValueError):
            kvr.verify_drafts(x, d, torch.zeros(S, T, dtype=torch.int32),
                              torch.zeros(S, T), torch.ones(S, V))


def test_strides_of_rows_that_do_not_overlap():
    V = 33
    wide = torch.zeros(3, 4, V + 5)
    assert kvr._logit_rows(wide[..., :V], "target") == V + 5
    assert kvr._logit_rows(wide[:, :, 2:2 + V], "target") == V + 5
    assert kvr._logit_rows(wide[:1, :1, :V], "target") >= V
    assert kvr._logit_rows(torch.zeros(3, 1, V), "target") == V
    assert kvr._logit_rows(torch.zeros(V).expand(1, 1, V), "target") == V
    assert kvr._logit_rows(torch.zeros(6, 1).expand(6, 1)[:, None], "x") == 1
    with pytest.raises(ValueError):
        kvr._logit_rows(wide[:, ::2, :V][:, :, ::2], "target")
    with pytest.raises(ValueError):
        kvr._logit_rows(wide.transpose(0, 1)[..., :V], "target")
