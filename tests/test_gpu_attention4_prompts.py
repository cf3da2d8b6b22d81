"""kd.attention_4bit for whole prompts and pieces of them: hundreds of rows a sequence."""

import pytest
import torch

from test_gpu_attention4 import BF16, F16, Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kd():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2609_11687_gb300 import build
    build.build()
    from paper_2609_11687_gb300 import kashin
    return kashin


@pytest.mark.parametrize("dt", [F16, BF16])
@pytest.mark.parametrize("lengths,counts,hq,hk,d,group", [([300, 200, 1], [300, 200, 1], 8, 2, 64, 32), ([500], [500], 4, 4, 128, 64),
                                                          ([400, 90, 0, 130], [64, 90, 1, 7], 8, 2, 128, 128), ([150], [150], 8, 1, 256, 64),
                                                          ([70, 700], [70, 33], 10, 2, 80, 32), ([33] * 40, [33] * 40, 4, 2, 96, 64)])
def test_prompts(kd, lengths, counts, hq, hk, d, group, dt):
    for longest in (None, 0):  # the largest length, a hint that says nothing
        c = Case(kd, lengths, counts, hq, hk, d, group=group, dt=dt, spare=1, longest=longest)
        assert kd.attention_4bit_workspace(c.cache, c.seqs, hq) == 0
        c.check(kd)
    c.check(kd, window=50)
    c.check(kd, causal=False)
