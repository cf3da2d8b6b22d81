"""kd.rmsnorm against its formula in 64 bits.

Tolerances, with u = 2^-24: the sum of squares adds at most 32 terms in a thread, 5 + 4 in
the tree and rounds each square once (all terms positive: at most 46 u relative), so its
root is off by 23 u; the mean, eps, root, reciprocal, h and the two products round once
each: 32 u |y| bounds y, 40 u the scale (one division more).  An output in fewer bits adds
half a unit of its type; q is within half a unit of e4m3 (2^-4 relative, 2^-10 below its
normal range) of y / scale."""

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
# half a unit of a rounded output: relative, and absolute below the normal range
HALF_UNIT = {torch.float32: (0.0, 2.0 ** -149), torch.float16: (torch.finfo(torch.float16).eps / 2, 2.0 ** -25),
             torch.bfloat16: (torch.finfo(torch.bfloat16).eps / 2, 2.0 ** -134)}


@pytest.fixture(scope="module")
def kd():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2609_11687_gb300 import build
    build.build()
    from paper_2609_11687_gb300 import kashin
    return kashin


def _rows(g, rows, n, dt, off=0, pad=0):
    """(rows, n) values at a row stride of n + pad, `off` elements into their buffer."""
    buf = torch.empty(off + rows * (n + pad), dtype=dt, device="cuda")
    v = buf[off:].view(rows, n + pad)[:, :n] if rows else torch.empty((0, n), dtype=dt, device="cuda")
    v.copy_(torch.randn((rows, n), generator=g, device="cuda") * 2)
    return v


def _check(kd, x, w, residual, r, eps):
    x64 = x.double()
    h = x64 if residual is None else x64 + residual.double()
    y = h / (h.square().mean(1, keepdim=True) + eps).sqrt() * w.double()
    if r.residual is not None:
        want = x.float() if residual is None else x.float() + residual.float()
        assert torch.equal(r.residual, want.to(x.dtype))
    if r.y is not None:
        rel, least = HALF_UNIT[r.y.dtype]
        assert ((r.y.double() - y).abs() <= (rel + 33 * U) * y.abs() + least).all()
    if r.q is not None:
        amax = y.abs().amax(1)
        scale = torch.where(amax < 2.0 ** -100, torch.ones_like(amax), amax / 448)
        assert ((r.scale.double() - scale).abs() <= 40 * U * scale).all()
        v = y / r.scale.double()[:, None]
        assert ((r.q.double() - v).abs() <= torch.clamp((2.0 ** -4 + 80 * U) * v.abs(), min=1.01 * 2.0 ** -10)).all()


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,n", [(1, 1), (3, 7), (1, 8), (5, 16), (33, 250), (2, 256), (7, 1000), (1, 4096), (9, 4096), (4, 5003),
                                    (3, 8192), (2, 11008), (3, 16383), (2, 16384)])
def test_against_64_bits(kd, dt, rows, n):
    g = torch.Generator(device="cuda").manual_seed(rows * 100003 + n)
    x, res = _rows(g, rows, n, dt), _rows(g, rows, n, dt)
    w = (1 + 0.2 * torch.randn(n, generator=g, device="cuda")).to(dt)
    for residual in (None, res):
        for wt in (w, w.float()):
            out = kd.Normed(q=torch.empty((rows, n), dtype=torch.float8_e4m3fn, device="cuda"),
                            scale=torch.empty(rows, device="cuda"),
                            y=torch.empty((rows, n), device="cuda", dtype=torch.float32),
                            residual=None if residual is None else torch.empty_like(x))
            _check(kd, x, wt, residual, kd.rmsnorm(x, wt, 1e-5, residual=residual, out=out), 1e-5)
    _check(kd, x, w, res, kd.rmsnorm(x, w, 1e-6, residual=res), 1e-6)


@pytest.mark.parametrize("ydt", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n", [512, 777])
def test_y_alone_in_each_type(kd, ydt, n):
    g = torch.Generator(device="cuda").manual_seed(n)
    x = _rows(g, 6, n, torch.bfloat16)
    w = torch.randn(n, generator=g, device="cuda").to(torch.bfloat16)
    r = kd.rmsnorm(x, w, out=kd.Normed(y=torch.empty((6, n), dtype=ydt, device="cuda")))
    assert r.q is None and r.scale is None
    _check(kd, x, w, None, r, 1e-5)


@pytest.mark.parametrize("off,pad", [(0, 8), (0, 3), (1, 7), (8, 40)])
def test_strides_and_alignment(kd, off, pad):
    """Rows at strides past n, aligned or not, give the contiguous rows' bits and leave the
    gap between rows alone."""
    g = torch.Generator(device="cuda").manual_seed(3)
    rows, n, dt = 5, 640, torch.float16
    x, res = _rows(g, rows, n, dt, off, pad), _rows(g, rows, n, dt, off, pad)
    w = torch.randn(n, generator=g, device="cuda").to(dt)
    ref = kd.rmsnorm(x.contiguous(), w, residual=res.contiguous())
    qb = torch.full((rows, n + pad), 7, dtype=torch.uint8, device="cuda")
    yb = torch.full((rows, n + pad), 7.0, dtype=dt, device="cuda")
    rb = torch.full((rows, n + pad), 7.0, dtype=dt, device="cuda")
    out = kd.Normed(q=qb.view(torch.float8_e4m3fn)[:, :n], scale=torch.empty(rows, device="cuda"), y=yb[:, :n], residual=rb[:, :n])
    kd.rmsnorm(x, w, residual=res, out=out)
    # element accesses sum a row's squares in another order
    assert torch.equal(rb[:, :n], ref.residual)
    _check(kd, x, w, res, out, 1e-5)
    assert (qb[:, n:] == 7).all() and (yb[:, n:] == 7).all() and (rb[:, n:] == 7).all()


def test_in_place_residual_and_y(kd):
    g = torch.Generator(device="cuda").manual_seed(4)
    x, res = _rows(g, 4, 1024, torch.bfloat16), _rows(g, 4, 1024, torch.bfloat16)
    w = torch.randn(1024, generator=g, device="cuda").to(torch.bfloat16)
    ref = kd.rmsnorm(x, w, residual=res, out=kd.Normed(y=torch.empty_like(x), residual=torch.empty_like(x)))
    x2, r2 = x.clone(), res.clone()
    kd.rmsnorm(x2, w, residual=r2, out=kd.Normed(y=x2, residual=r2))
    assert torch.equal(x2, ref.y) and torch.equal(r2, ref.residual)


def test_special_rows(kd):
    """A row of zeros, rows that hold NaN or an infinity, a row whose squares overflow; their
    neighbours are untouched."""
    n = 512
    x = torch.ones((6, n), device="cuda")
    x[1] = 0
    x[2, 5] = float("nan")
    x[3, 500] = float("inf")
    x[4] = 1e25
    r = kd.rmsnorm(x, torch.ones(n, device="cuda"), 0.0 + 1e-5,
                   out=kd.Normed(q=torch.empty((6, n), dtype=torch.float8_e4m3fn, device="cuda"),
                                 scale=torch.empty(6, device="cuda"), y=torch.empty((6, n), device="cuda")))
    assert (r.q[1].float() == 0).all() and r.scale[1] == 1 and (r.y[1] == 0).all()
    for k in (2, 3, 4):
        assert r.scale[k].isnan() and r.q[k].float().isnan().all() and r.y[k].isnan().all()
    for k in (0, 5):
        _check(kd, x[k:k + 1], torch.ones(n, device="cuda"), None, kd.Normed(q=r.q[k:k + 1], scale=r.scale[k:k + 1], y=r.y[k:k + 1]), 1e-5)


def test_large_offsets(kd):
    """A row stride that takes rows past 2^32 bytes and 2^31 elements."""
    ld = 2 ** 30 + 8
    buf = torch.empty(2 * ld + 4096, dtype=torch.float16, device="cuda")
    x = buf.as_strided((3, 4096), (ld, 1))
    x.copy_(torch.randn((3, 4096), device="cuda"))
    w = torch.ones(4096, dtype=torch.float16, device="cuda")
    _check(kd, x, w, None, kd.rmsnorm(x, w), 1e-5)


def test_other_stream_empty_and_refusals(kd):
    g = torch.Generator(device="cuda").manual_seed(6)
    x = _rows(g, 3, 768, torch.float16)
    w = torch.ones(768, dtype=torch.float16, device="cuda")
    ref = kd.rmsnorm(x, w)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    a = kd.rmsnorm(x, w, stream=s)
    with torch.cuda.stream(s):
        b = kd.rmsnorm(x, w)
    s.synchronize()
    for r in (a, b):
        assert torch.equal(r.q.view(torch.uint8), ref.q.view(torch.uint8)) and torch.equal(r.scale, ref.scale)
    e = kd.rmsnorm(x[:0], w)
    assert e.q.shape == (0, 768) and e.scale.shape == (0,)
    with pytest.raises(ValueError, match="residual"):
        kd.rmsnorm(x, w, out=kd.Normed(y=torch.empty_like(x), residual=torch.empty_like(x)))
    with pytest.raises(ValueError, match="shape"):
        kd.rmsnorm(x, w[:-1])
    with pytest.raises(ValueError, match="dtype"):
        kd.rmsnorm(x, w.bfloat16())
    with pytest.raises(ValueError, match="wants"):
        kd.rmsnorm(x, w, out=kd.Normed())
    with pytest.raises(ValueError, match="inner stride"):
        kd.rmsnorm(x.t().contiguous().t(), w)
    with pytest.raises(kd.KashinError):
        kd.rmsnorm(torch.zeros((1, 16385), device="cuda"), torch.zeros(16385, device="cuda"))
