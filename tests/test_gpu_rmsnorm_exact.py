"""kd.rmsnorm's 8-bit rows against its own fp32 rows, bit for bit: scale is max |y| / 448 and
q is e4m3(y / scale), of which every step is one IEEE operation; and rows whose products of
value and weight leave fp32's range although y does not."""

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module")
def kd():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2609_11687_gb300 import build
    build.build()
    from paper_2609_11687_gb300 import kashin
    return kashin


def _all(kd, x, w, eps=1e-5, residual=None):
    rows, n = x.shape
    out = kd.Normed(q=torch.empty((rows, n), dtype=torch.float8_e4m3fn, device="cuda"), scale=torch.empty(rows, device="cuda"),
                    y=torch.empty((rows, n), device="cuda"), residual=None if residual is None else torch.empty_like(x))
    return kd.rmsnorm(x, w, eps, residual=residual, out=out)


def _q_of(y):
    """Scale and e4m3 rows of fp32 rows (a division by a tensor: by a number torch may multiply)."""
    amax = y.abs().amax(1)
    scale = torch.where(amax < 2.0 ** -100, torch.ones_like(amax), amax / torch.full_like(amax, 448.0))
    return scale, (y / scale[:, None]).to(torch.float8_e4m3fn)


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,n", [(1, 1), (5, 33), (40, 777), (512, 4096), (700, 640), (64, 5003), (9, 16384)])
def test_q_and_scale_follow_from_y(kd, dt, rows, n):
    g = torch.Generator(device="cuda").manual_seed(rows + n)
    x, res = (torch.randn((2, rows, n), generator=g, device="cuda") * 2).to(dt)
    w = (1 + 0.2 * torch.randn(n, generator=g, device="cuda")).to(dt)
    for wt in (w, w.float()):
        for residual in (None, res):
            r = _all(kd, x, wt, residual=residual)
            scale, q = _q_of(r.y)
            assert torch.equal(r.scale, scale)
            assert torch.equal(r.q.view(torch.uint8), q.view(torch.uint8))


@pytest.mark.parametrize("n", [256, 1001])
@pytest.mark.parametrize("size,weight", [(3e17, 1e25), (1e15, 1e30), (3e-18, 1e-20), (1.0, 1e-36)])
def test_products_outside_the_range(kd, n, size, weight):
    """|x w| above 3e38 or far below 1e-38, y within: scale and q are y's.  Bounds: the sum of
    squares of at most 1024 values, eps = 0 (33 u of y, as for any row); subnormals of y by
    their spacing."""
    g = torch.Generator(device="cuda").manual_seed(n)
    x = torch.randn((6, n), generator=g, device="cuda") * size
    w = (1 + torch.rand(n, generator=g, device="cuda")) * weight
    r = _all(kd, x, w, eps=0.0)
    want = x.double() / x.double().square().mean(1, keepdim=True).sqrt() * w.double()
    assert torch.isfinite(r.y).all() and torch.isfinite(r.scale).all()
    assert ((r.y.double() - want).abs() <= 33 * U * want.abs() + 2.0 ** -149).all()
    scale, q = _q_of(r.y)
    assert torch.equal(r.scale, scale) and torch.equal(r.q.view(torch.uint8), q.view(torch.uint8))
    assert weight < 1e-30 or r.q.float().abs().amax() == 448
