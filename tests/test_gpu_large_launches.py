"""Calls whose items are more than one launch has threads for: every one is answered."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def P():
    import paper_2603_04135_amd as P
    P.load()
    assert torch.cuda.is_available(), "these tests need the GPU"
    return P


def test_gather_of_more_than_2_to_the_32_items(P):
    period = 1000
    src = torch.rand(period, device=DEV)
    idx = torch.arange(period - 1, -1, -1, device=DEV, dtype=torch.int32).repeat(2 ** 32 // period + 1)
    assert idx.numel() > 2 ** 32
    out = P.dppo_gather_f32(idx, src)
    assert (out.view(-1, period) == src.flip(0)).all()


def test_token_norm_of_more_than_2_to_the_26_groups(P):
    Q = 2 ** 26 + 5
    lengths = torch.arange(Q, device=DEV, dtype=torch.int32).remainder_(7)
    coef = torch.rand(Q, device=DEV)
    out = P.dppo_token_norm_coef(coef[:, None], lengths[:, None])[:, 0]
    want = coef * torch.where(lengths > 0, 1.0 / lengths.double(), torch.zeros((), dtype=torch.float64, device=DEV)).float()
    assert torch.equal(out, want)
