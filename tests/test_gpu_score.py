"""The output head's whole path (kd.rmsnorm -> kd.matmul_4bit -> kd.token_logprobs) as a
program runs it: against 64 bits from the path's own 8-bit rows, in a CUDA graph, and the
example."""

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


def _setup(rows, hidden, vocab, dt):
    g = torch.Generator(device="cuda").manual_seed(rows + vocab)

    def randn(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    head = (randn(vocab, hidden) * 0.1).to(dt)
    norm = (1 + 0.1 * randn(hidden)).to(dt)
    return head, norm, randn(rows, hidden).to(dt), randn(rows, hidden).to(dt), torch.randint(0, vocab, (rows,), generator=g, device="cuda")


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rows,hidden,vocab", [(1, 768, 5003), (5, 1000, 4001), (40, 512, 1000)])
def test_output_head(kd, dt, rows, hidden, vocab):
    """The logits differ from 64 bits by the product's fp32 sums (2e-5 of a row's largest
    is far above them), a log probability by twice the largest such difference more."""
    from paper_2609_11687_gb300.score import OutputHead
    head, norm, x, res, ids = _setup(rows, hidden, vocab, dt)
    h = OutputHead(norm, head, group=64)
    r = kd.rmsnorm(x, norm, 1e-5, residual=res)
    want = (r.q.double() * r.scale.double()[:, None]) @ kd.dequantise_4bit(h.head).double().t()
    tol = 2e-5 * want.abs().amax(1)
    assert ((h.logits(x, res).double() - want).abs() <= tol[:, None]).all()
    s = h.score(x, ids, res, top=3)
    lp = want.log_softmax(1)
    assert ((s.logprobs[:, 0].double() - lp.gather(1, ids[:, None])[:, 0]).abs() <= 3 * tol + 1e-5).all()
    assert ((s.top_logprobs.double() - lp.topk(3).values).abs() <= 3 * tol[:, None] + 1e-5).all()


def test_output_head_in_a_graph(kd):
    """One decoded token's step captured once and replayed on new rows gives the eager bits."""
    from paper_2609_11687_gb300.score import OutputHead
    head, norm, x, res, ids = _setup(2, 768, 3000, torch.float16)
    h = OutputHead(norm, head)
    h.score(x, ids, res, top=5)
    torch.cuda.synchronize()
    gr = torch.cuda.CUDAGraph()
    with torch.cuda.graph(gr):
        out = h.score(x, ids, res, top=5)
    x.copy_(torch.randn_like(x))
    gr.replay()
    torch.cuda.synchronize()
    ref = h.score(x, ids, res, top=5)
    for a, b in zip(vars(out).values(), vars(ref).values()):
        assert torch.equal(a, b)


def test_example(kd):
    """Fewer bits score no better than the head that the tokens were drawn from (the drawn
    tokens' own noise allowed for), and 4 bits stay close to it."""
    from paper_2609_11687_gb300 import score
    out = score.main(["--rows", "256", "--hidden", "512", "--vocab", "2000"])
    assert out["4 bits"] < 1.2 * out["dense fp16"] and out["dense fp16"] < 1.05 * out["2-bit planes"]
    assert all(1 < v < 2000 for v in out.values())
