"""Calls with ``stream=``: what they allocate must not be memory that work still pending on the
current stream reads, and what they return must not be given out again while it is read."""

import pytest
import torch

pytestmark = pytest.mark.gpu

PENDING = 20_000_000  # cycles of a kernel that keeps the current stream back: about 10 ms


@pytest.fixture(scope="module")
def kd():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2609_11687_gb300 import build
    build.build()
    from paper_2609_11687_gb300 import kashin
    return kashin


def _tensors(out):
    if isinstance(out, torch.Tensor):
        return [out]
    if hasattr(out, "codes") and hasattr(out, "scales"):
        return [t for t in (out.codes, out.scales, out.zeros) if t is not None]
    return [t for t in vars(out).values() if t is not None]


def _bytes(t):
    return t.contiguous().view(torch.uint8) if t.dim() and t.numel() else t


def _calls(kd):
    """name -> call(stream); the inputs are there when this returns."""
    from paper_2609_11687_gb300.score import OutputHead
    g = torch.Generator(device="cuda").manual_seed(1)

    def randn(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    x, res, norm = randn(40, 1024).half(), randn(40, 1024).half(), randn(1024).half()
    weight = randn(2000, 1024).half() * 0.1
    w4 = kd.quantise_4bit(weight, 64, zeros=True)
    logits, ids = randn(40, 2000), torch.randint(0, 2000, (40, 2), generator=g, device="cuda")
    head = OutputHead(norm, w4)
    torch.cuda.synchronize()
    return {
        "rmsnorm": lambda s: kd.rmsnorm(x, norm, residual=res, stream=s),
        "quantise_4bit": lambda s: kd.quantise_4bit(weight, 64, zeros=True, stream=s),
        "dequantise_4bit": lambda s: kd.dequantise_4bit(w4, stream=s),
        "matmul_4bit": lambda s: kd.matmul_4bit(w4, x, stream=s),
        "token_logprobs": lambda s: kd.token_logprobs(logits, ids, 5, stream=s),
        "OutputHead.logits": lambda s: head.logits(x, res, stream=s),
        "OutputHead.score": lambda s: head.score(x, ids, res, top=5, stream=s),
    }


NAMES = ["rmsnorm", "quantise_4bit", "dequantise_4bit", "matmul_4bit", "token_logprobs", "OutputHead.logits", "OutputHead.score"]
# of every size that a call above allocates, scratch between its kernels included
SIZES = [40 * 1024, 40 * 1024 * 2, 40 * 4, 2000 * 512, 2000 * 16 * 2, 2000 * 16, 2000 * 1024 * 4, 40 * 2000 * 4, 40 * 2 * 4, 40 * 5 * 8,
         40 * 5 * 4, 1 << 21, 1 << 21]


@pytest.mark.parametrize("name", NAMES)
def test_outputs_are_not_memory_still_read(kd, name):
    call = _calls(kd)[name]
    want = [_bytes(t).clone() for t in _tensors(call(None))]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    freed = [torch.full((size,), 7, dtype=torch.uint8, device="cuda") for size in SIZES for _ in range(3)]
    torch.cuda.synchronize()
    torch.cuda._sleep(PENDING)
    read = [t.clone() for t in freed]  # not before the kernel above has ended
    places = {t.data_ptr() for t in freed}
    del freed
    out = call(side)
    assert not places & {t.data_ptr() for t in _tensors(out)}
    torch.cuda.synchronize()
    assert all((t == 7).all() for t in read)
    for a, b in zip(_tensors(out), want):
        assert torch.equal(_bytes(a), b)


@pytest.mark.parametrize("name", NAMES)
def test_a_dropped_result_is_kept_until_it_is_read(kd, name):
    call = _calls(kd)[name]
    want = [_bytes(t).clone() for t in _tensors(call(None))]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    out = call(side)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda._sleep(PENDING)
    read = [_bytes(t).clone() for t in _tensors(out)]
    sizes = [t.numel() * t.element_size() for t in _tensors(out)]
    del out
    with torch.cuda.stream(side):
        over = [torch.full((n,), 9, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(3)]
    torch.cuda.synchronize()
    assert len(over) == 3 * len(sizes)
    for a, b in zip(read, want):
        assert torch.equal(a, b)


def test_a_step_on_another_stream_in_a_graph(kd):
    """Captured with its work on a second stream, a step still gives the eager bits."""
    call = _calls(kd)["OutputHead.score"]
    want = [t.clone() for t in _tensors(call(None))]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    gr = torch.cuda.CUDAGraph()
    with torch.cuda.graph(gr):
        side.wait_stream(torch.cuda.current_stream())
        out = call(side)
        torch.cuda.current_stream().wait_stream(side)
    gr.replay()
    torch.cuda.synchronize()
    for a, b in zip(_tensors(out), want):
        assert torch.equal(a, b)
