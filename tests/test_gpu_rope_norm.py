"""kd.rope's head norm to the bit, where fp32's sums of squares are exact."""

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kd():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2609_11687_gb300 import build
    build.build()
    from paper_2609_11687_gb300 import kashin
    return kashin


@pytest.mark.parametrize("eps", [0.0, 1e-6, 0.5])
@pytest.mark.parametrize("d,pad", [(128, 0), (64, 0), (16, 0), (128, 3)])  # the last pair by pair
def test_the_norms_factor_is_a_root_and_a_quotient(kd, d, pad, eps):
    """Whole numbers up to 255: their squares add up exactly in any order, d is a power of two, and at position 0 nothing
    turns.  Then x (1 / sqrt(mean + eps)) w has five roundings, each of an operation that IEEE defines."""
    g = torch.Generator().manual_seed(d)
    x = torch.randint(-255, 256, (999, 2, d), generator=g).float()
    w = 1 + 0.1 * torch.randn(d, generator=g)
    mean = x.square().sum(2, keepdim=True) * (1.0 / d)
    want = x * (torch.ones(()) / torch.sqrt(mean + torch.tensor(eps, dtype=torch.float32))) * w
    wide = torch.zeros((999, 2, d + pad), device="cuda")
    wide[..., :d] = x.cuda()
    zero = torch.zeros(999, dtype=torch.int64, device="cuda")
    q, k = wide[..., :d], x.cuda()
    yq, yk = kd.rope(q, k, zero, kd.Rotation(d), w.cuda(), w.cuda(), eps=eps)
    assert torch.equal(yq.cpu(), want) and torch.equal(yk.cpu(), want)
