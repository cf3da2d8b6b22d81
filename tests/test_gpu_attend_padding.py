"""Rows of no sequence in an attention step's batch: whatever they hold, the other rows and the cache keep their bits."""

import math

import pytest
import torch

from test_gpu_attend import _sequences, _step

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kd():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2609_11687_gb300 import build
    build.build()
    from paper_2609_11687_gb300 import kashin
    return kashin


@pytest.mark.parametrize("counts,padding", [([1, 1, 1], 5), ([3, 0, 2], 11), ([20, 1, 7], 30)])
def test_padding_touches_nothing(kd, counts, padding):
    results = []
    for held in (0.0, 1.0, math.nan, math.inf):
        step, randn = _step(kd, 256, 4, 2, 64, torch.bfloat16)
        table = torch.arange(36, device="cuda").view(3, 12).int()
        seqs, positions = _sequences(kd, [40, 33, 50], counts, 16, table)
        rows = sum(counts)
        x = randn(rows + padding, 256).bfloat16()
        x[rows:] = held
        at = torch.cat((positions, torch.full((padding,), -3, device="cuda")))
        junk = torch.full((rows + padding, 4, 64), held, dtype=torch.bfloat16, device="cuda")  # what a new tensor may be made of
        del junk
        y, residual = step.step(x, at, seqs, residual=x)
        results.append((y[:rows], residual[:rows], *(t.clone() for t in (step.cache.k_codes, step.cache.k_scales, step.cache.v_codes, step.cache.v_scales))))
    for other in results[1:]:
        for a, b in zip(results[0], other):
            assert torch.equal(a, b)
    assert torch.isfinite(results[0][0]).all()
