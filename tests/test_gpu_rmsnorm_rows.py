"""kd.rmsnorm on more rows than are resident at a time, so that every CTA walks several, in
place and not, against the formula in 64 bits.

Tolerances, with u = 2^-24: a thread adds at most 16 squares (fused: one rounding each), five
levels of shuffles and at most 32 warps follow, all terms positive: the sum of squares is off by
53 u, its root by 26.5; the mean and eps round within it (1 u together), root, reciprocal, h
(twice: in the root too) and the two products once each: 34 u |y|.  An output in fewer bits adds
half a unit of its type; q is e4m3(y / scale) of the rounded y, half a unit of e4m3 and the
34 u and the scale's 35 more."""

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF_UNIT = {torch.float32: (0.0, 2.0 ** -149), torch.float16: (torch.finfo(torch.float16).eps / 2, 2.0 ** -25),
             torch.bfloat16: (torch.finfo(torch.bfloat16).eps / 2, 2.0 ** -134)}


@pytest.fixture(scope="module")
def kd():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2609_11687_gb300 import build
    build.build()
    from paper_2609_11687_gb300 import kashin
    return kashin


def _check(x, w, residual, r, eps=1e-5):
    """x and residual are copies from before the call."""
    h = x.double() if residual is None else x.double() + residual.double()
    y = h / (h.square().mean(1, keepdim=True) + eps).sqrt() * w.double()
    if residual is not None:
        assert torch.equal(r.residual, (x.float() + residual.float()).to(x.dtype))
    if r.y is not None:
        rel, least = HALF_UNIT[r.y.dtype]
        assert ((r.y.double() - y).abs() <= (rel + 35 * U) * y.abs() + least).all()
    if r.q is not None:
        scale = y.abs().amax(1) / 448
        assert ((r.scale.double() - scale).abs() <= 36 * U * scale).all()
        v = y / r.scale.double()[:, None]
        assert ((r.q.double() - v).abs() <= torch.clamp((2.0 ** -4 + 72 * U) * v.abs(), min=1.01 * 2.0 ** -10)).all()


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,n", [(2048, 4096), (1531, 4096), (9001, 250), (6007, 640), (20011, 72), (700, 11008), (333, 5003),
                                    (1000, 5003), (1300, 1001), (500, 16384), (400, 16383), (609, 257)])
def test_many_rows(kd, dt, rows, n):
    g = torch.Generator(device="cuda").manual_seed(rows * 7 + n)
    # rows of different sizes: one row's sum in another's place would show
    size = torch.exp(torch.randn((rows, 1), generator=g, device="cuda"))
    x, res = ((torch.randn((2, rows, n), generator=g, device="cuda") * size) * 2).to(dt)
    w = (1 + 0.2 * torch.randn(n, generator=g, device="cuda")).to(dt)
    for wt in (w, w.float()):
        out = kd.Normed(q=torch.empty((rows, n), dtype=torch.float8_e4m3fn, device="cuda"), scale=torch.empty(rows, device="cuda"),
                        y=torch.empty((rows, n), device="cuda"), residual=torch.empty_like(x))
        _check(x, wt, res, kd.rmsnorm(x, wt, residual=res, out=out))
    # nothing but 8-bit rows, of x alone
    _check(x, w, None, kd.rmsnorm(x, w))
    # the sum in the residual's place, the normed rows in x's
    x2, r2 = x.clone(), res.clone()
    _check(x, w, res, kd.rmsnorm(x2, w, residual=r2, out=kd.Normed(y=x2, residual=r2)))
    # the same bits again
    again = kd.rmsnorm(x, w, residual=res, out=kd.Normed(y=torch.empty_like(x), residual=torch.empty_like(x)))
    assert torch.equal(again.y, x2) and torch.equal(again.residual, r2)


@pytest.mark.parametrize("rows,n", [(3000, 512), (1500, 777)])
def test_special_rows_among_many(kd, rows, n):
    """Rows that hold NaN or an infinity, and rows of zeros, leave the rows that their CTA
    takes before and after them alone."""
    g = torch.Generator(device="cuda").manual_seed(n)
    x = torch.randn((rows, n), generator=g, device="cuda").bfloat16()
    w = torch.ones(n, device="cuda").bfloat16()
    x[::7, n // 2] = float("nan")
    x[3::11, n - 1] = float("inf")
    x[5::13] = 0
    out = kd.Normed(q=torch.empty((rows, n), dtype=torch.float8_e4m3fn, device="cuda"), scale=torch.empty(rows, device="cuda"),
                    y=torch.empty((rows, n), device="cuda"))
    r = kd.rmsnorm(x, w, out=out)
    bad = ~torch.isfinite(x.float()).all(1)
    zero = (x == 0).all(1)
    fine = ~bad & ~zero
    assert r.y[bad].isnan().all() and r.scale[bad].isnan().all() and r.q[bad].float().isnan().all()
    assert (r.y[zero] == 0).all() and (r.scale[zero] == 1).all() and (r.q[zero].float() == 0).all()
    _check(x[fine], w, None, kd.Normed(q=r.q[fine], scale=r.scale[fine], y=r.y[fine]))
