"""Decomposition, reconstruction, P and the 2-bit products with ``stream=``: what they allocate,
scratch included, must not be memory that work still pending on the current stream reads."""

import types

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
    if isinstance(out, (list, tuple)):
        return [t for o in out for t in _tensors(o)]
    return [t for t in vars(out).values() if t is not None]


def _calls(kd):
    g = torch.Generator(device="cuda").manual_seed(2)
    w = (torch.randn((48, 256), generator=g, device="cuda") * 0.02).half()
    x = torch.randn((4, 256), generator=g, device="cuda")
    d, xp = kd.decompose(w, 8, 3), kd.apply_p(x, 3)
    x16, xp16 = x.half(), xp.half()
    ws = kd.prepare_p(256, [3])
    torch.cuda.synchronize()
    return {
        "decompose": lambda s: kd.decompose(w, 8, 3, factors=True, stream=s),
        "decompose_batch": lambda s: kd.decompose_batch([w, w], 8, [3, 4], coeffs=True, stream=s),
        "matmul_2bit": lambda s: kd.matmul_2bit(d, x, xp, stream=s),
        "matmul_2bit_f16": lambda s: kd.matmul_2bit_f16(d, x16, xp16, stream=s),
        "apply_p": lambda s: kd.apply_p(x, 3, stream=s),
        "apply_p_batch": lambda s: kd.apply_p_batch([x, x], [3, 4], stream=s),
        "apply_p_prepared": lambda s: kd.apply_p_prepared([x], ws, stream=s),
        "dequantise": lambda s: kd.dequantise(d.codes_u, d.centres_u, 256, stream=s),
        "rht": lambda s: kd.rht(x, 3, stream=s),
        "reconstruct": lambda s: kd.reconstruct(d, 256, 3, stream=s),
        "reconstruct_batch": lambda s: kd.reconstruct_batch([d, d], 256, [3, 3], stream=s),
    }


@pytest.mark.parametrize("name", ["decompose", "decompose_batch", "matmul_2bit", "matmul_2bit_f16", "apply_p", "apply_p_batch", "apply_p_prepared",
                                  "dequantise", "rht", "reconstruct", "reconstruct_batch"])
def test_outputs_are_not_memory_still_read(kd, name):
    call = _calls(kd)[name]
    want = [t.clone() for t in _tensors(call(None))]
    sizes = {t.numel() * t.element_size() for t in want} | {kd.kd_workspace_size(256), kd.kd_workspace_size_batch(256, 2)}
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    freed = [torch.full((size,), 7, dtype=torch.uint8, device="cuda") for size in sizes for _ in range(8)]
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
        assert torch.equal(a, b)


def test_a_holder_of_a_bare_handle(kd):
    """Any object with a stream's handle will do."""
    call = _calls(kd)["reconstruct"]
    want = call(None)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    out = call(types.SimpleNamespace(cuda_stream=side.cuda_stream))
    side.synchronize()
    assert torch.equal(out, want)
