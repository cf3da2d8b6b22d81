"""The output head on 16-bit rows, and the example's lines: heads are compared on the same rows."""

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


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rows", [1, 12, 40])
def test_16_bit_rows(kd, dt, rows):
    """The same bits as norm and product one by one, with and without a residual."""
    from paper_2609_11687_gb300.score import OutputHead
    g = torch.Generator(device="cuda").manual_seed(rows)
    x, res = torch.randn((2, rows, 512), generator=g, device="cuda").to(dt)
    norm = (1 + 0.1 * torch.randn(512, generator=g, device="cuda")).to(dt)
    h = OutputHead(norm, torch.randn((1000, 512), generator=g, device="cuda").to(dt), eight_bits=False)
    for residual in (None, res):
        r = kd.rmsnorm(x, norm, residual=residual, out=kd.Normed(y=torch.empty_like(x)))
        assert torch.equal(h.logits(x, residual), kd.matmul_4bit(h.head, r.y))
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    a = h.logits(x, res, stream=s)
    s.synchronize()
    assert torch.equal(a, h.logits(x, res))


def test_the_example_compares_heads_on_the_same_rows(kd):
    """Its lines again from the same draws: the dense and both coded heads read fp16 rows."""
    from paper_2609_11687_gb300 import score
    out = score.main(["--rows", "200", "--hidden", "512", "--vocab", "1500", "--seed", "3"])
    assert list(out) == ["dense fp16", "4 bits", "4 bits, 8-bit rows", "2-bit planes"]
    g = torch.Generator(device="cuda").manual_seed(3)

    def randn(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    head = (randn(1500, 512) * 512 ** -0.5 * 3).half()
    norm = (1 + 0.1 * randn(512)).half()
    x, res = randn(200, 512).half(), randn(200, 512).half()
    r = kd.rmsnorm(x, norm, residual=res, out=kd.Normed(q=torch.empty(x.shape, dtype=torch.float8_e4m3fn, device="cuda"),
                                                        scale=torch.empty(200, device="cuda"), y=torch.empty_like(x)))
    dense = r.y @ head.t()
    ids = torch.multinomial(dense.float().softmax(1), 1, generator=g)
    w4 = kd.quantise_4bit(head)

    def perplexity(logits):
        return score.perplexity(kd.token_logprobs(logits, ids).logprobs)

    assert out["dense fp16"] == perplexity(dense)
    assert out["4 bits"] == perplexity(kd.matmul_4bit(w4, r.y))
    assert out["4 bits, 8-bit rows"] == perplexity(kd.matmul_4bit(w4, r.q, scale=r.scale))
