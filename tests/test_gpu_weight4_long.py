"""kd.matmul_4bit on 9 to 16 rows of inputs so long that the kernel for few rows has no room
for them: one pass over the weights all the same where there are many channels and the rows are
aligned, else two of eight rows; against the product in 64 bits.

Tolerance, with A = sum_i |s (c - z) x_i|: c - z and its products with x are exact; the tensor
cores' sums of a group of 64 (four or eight steps of 16 or 32 inputs) hold 22 bits of their
largest part: 8 * 2^-22 A; the fp32 sums over the groups and up to eight CTAs round once each:
(groups + 9) 2^-24 A."""

import ctypes

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


def _launches(call):
    """Kernels that call() puts on the current stream, by the nodes of its capture."""
    cudart = ctypes.CDLL("libcudart.so.13")
    stream = torch.cuda.Stream()
    graph, nodes = ctypes.c_void_p(), ctypes.c_size_t()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        handle = ctypes.c_void_p(stream.cuda_stream)
        assert cudart.cudaStreamBeginCapture(handle, 2) == 0  # relaxed
        call()
        assert cudart.cudaStreamEndCapture(handle, ctypes.byref(graph)) == 0
    assert cudart.cudaGraphGetNodes(graph, None, ctypes.byref(nodes)) == 0
    assert cudart.cudaGraphDestroy(graph) == 0
    return nodes.value


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16, torch.float8_e4m3fn])
@pytest.mark.parametrize("rows", [9, 16])
@pytest.mark.parametrize("m,n,ld", [(48, 40000, 40000), (300, 40001, 40001), (2559, 39999, 40000), (2560, 39999, 40000),
                                    (2560, 39999, 39999), (2700, 40000, 40016), (2700, 65536, 65536), (64, 65536, 65536)])
def test_passes(kd, dt, rows, m, n, ld):
    g = torch.Generator(device="cuda").manual_seed(rows + n)
    group = 64
    groups = -(-n // group)
    codes = torch.randint(-2 ** 31, 2 ** 31, (m, (n + 31) // 32 * 4), generator=g, device="cuda", dtype=torch.int64).to(torch.int32)
    scales = (torch.exp(torch.randn((m, groups), generator=g, device="cuda")) * 0.01).half()
    zeros = torch.randint(0, 16, (m, groups), generator=g, device="cuda").to(torch.uint8)
    w = kd.Weight4(codes, scales, zeros, n=n, group=group)
    x = torch.randn((rows, ld), generator=g, device="cuda").to(dt)[:, :n]
    y = torch.empty((rows, m), device="cuda")
    kd.matmul_4bit(w, x, out=y)
    torch.cuda.synchronize()
    assert _launches(lambda: kd.matmul_4bit(w, x, out=y)) == (1 if m >= 2560 and ld % 8 == 0 else 2)
    c = ((codes[:, :, None] >> torch.arange(0, 32, 4, device="cuda", dtype=torch.int32)) & 15).flatten(1)[:, :n].double()
    c -= zeros.double().repeat_interleave(group, 1)[:, :n]
    c *= scales.double().repeat_interleave(group, 1)[:, :n]
    want, mass = x.double() @ c.t(), x.double().abs() @ c.abs().t()
    assert ((y.double() - want).abs() <= (8 * 2.0 ** -22 + (groups + 9) * 2.0 ** -24) * mass).all()
