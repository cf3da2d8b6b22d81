"""4-bit weights with group scales: kd.quantise_4bit and kd.dequantise_4bit bit for bit
against their IEEE definition, kd.matmul_4bit against the product in 64 bits.

Tolerance of the product, per output, with A = sum_i |s| (c + z) |x_i| |xs|: the tensor
cores' sums hold at least 22 bits relative to a sum's largest part, a group takes at most
16 of them (8 mma of 16 inputs; for e4m3 4 of 32 with 4 for the zero point): 16 * 2^-22 A;
the fp32 sums over the groups round once per group and join (8 warps, 8 CTAs):
(groups + 18) 2^-24 A.  An output in fewer bits adds half a unit of its type."""

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

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


def _codes(w):
    """(m, n) codes of a Weight4 on the host."""
    words = w.codes.cpu().numpy().view(np.uint32)
    i = np.arange(w.n)
    return (words[:, i // 8] >> (4 * (i % 8)).astype(np.uint32)) & 15


def _random(kd, g, m, n, group, zeros, sdt):
    """A Weight4 of random codes; the codes past n are random too."""
    words = (n + 31) // 32 * 4
    groups = (n + group - 1) // group
    codes = torch.randint(-2 ** 31, 2 ** 31, (m, words), generator=g, device="cuda", dtype=torch.int64).to(torch.int32)
    scales = (torch.exp(torch.randn((m, groups), generator=g, device="cuda")) * 0.01).to(sdt)
    z = torch.randint(0, 16, (m, groups), generator=g, device="cuda").to(torch.uint8) if zeros else None
    return kd.Weight4(codes, scales, z, n=n, group=group)


def _dense(w):
    """The weights and s (c + z) in 64 bits, (m, n)."""
    which = np.arange(w.n) // w.group
    c = _codes(w).astype(np.float64)
    s = w.scales.double().cpu().numpy()[:, which]
    z = 8.0 if w.zeros is None else w.zeros.double().cpu().numpy()[:, which]
    return s * (c - z), np.abs(s) * (c + z)


def _check(w, x, scale, y):
    W, A = _dense(w)
    xs = 1.0 if scale is None else scale.double().cpu().numpy()[:, None]
    x64 = x.double().cpu().numpy() * xs
    want, mass = x64 @ W.T, np.abs(x64) @ A.T
    rel, least = HALF_UNIT[y.dtype]
    groups = -(-w.n // w.group)
    tol = (16 * 2.0 ** -22 + (groups + 18) * 2.0 ** -24) * mass + rel * np.abs(want) * 1.01 + least
    assert (np.abs(y.double().cpu().numpy() - want) <= tol).all()


def _x(g, rows, n, kind):
    x = torch.randn((rows, n), generator=g, device="cuda")
    x[:, :: max(2, n // 3)] *= 30
    if kind == "e4m3":
        s = x.abs().amax(1) / 448
        return (x / s[:, None]).to(torch.float8_e4m3fn), s
    return x.to({"f16": torch.float16, "bf16": torch.bfloat16}[kind]), None


KINDS = ["f16", "bf16", "e4m3"]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("rows,m,n,zeros", [
    (1, 1, 1, False), (1, 1, 31, True), (2, 33, 32, True), (3, 31, 33, False), (8, 16, 127, False), (9, 40, 129, True), (1, 4096, 1024, False),
    (16, 65, 1000, True), (17, 70, 2049, False), (32, 32, 4096, True), (33, 47, 640, False), (70, 100, 777, True)])
def test_product(kd, kind, group, rows, m, n, zeros):
    g = torch.Generator(device="cuda").manual_seed(rows + 1000 * m + 7 * n + group)
    w = _random(kd, g, m, n, group, zeros, torch.bfloat16 if m % 2 else torch.float16)
    x, s = _x(g, rows, n, kind)
    _check(w, x, s, kd.matmul_4bit(w, x, scale=s))


@pytest.mark.parametrize("kind,rows,m,n", [("f16", 1, 64, 16384), ("bf16", 5, 200, 11008), ("e4m3", 16, 40, 16384), ("bf16", 1, 16, 40000)])
def test_product_long(kd, kind, rows, m, n):
    """Long inputs: clusters of CTAs share a tile."""
    g = torch.Generator(device="cuda").manual_seed(n)
    w = _random(kd, g, m, n, 64, True, torch.float16)
    x, s = _x(g, rows, n, kind)
    _check(w, x, s, kd.matmul_4bit(w, x, scale=s))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("odt", [torch.float16, torch.bfloat16])
def test_product_16_bit_output(kd, kind, odt):
    g = torch.Generator(device="cuda").manual_seed(11)
    w = _random(kd, g, 96, 512, 128, False, torch.float16)
    x, s = _x(g, 4, 512, kind)
    y = kd.matmul_4bit(w, x, scale=s, out_dtype=odt)
    assert y.dtype == odt
    _check(w, x, s, y)


@pytest.mark.parametrize("kind", KINDS)
def test_rows_alone_and_together_and_twice(kd, kind):
    """A row's result has the same bits alone, in a batch (within one tile count) and again."""
    g = torch.Generator(device="cuda").manual_seed(12)
    w = _random(kd, g, 150, 3000, 64, True, torch.float16)
    x, s = _x(g, 8, 3000, kind)
    y = kd.matmul_4bit(w, x, scale=s)
    assert torch.equal(y, kd.matmul_4bit(w, x, scale=s))
    for r in (0, 3, 7):
        assert torch.equal(y[r:r + 1], kd.matmul_4bit(w, x[r:r + 1], scale=None if s is None else s[r:r + 1]))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("off,pad", [(0, 16), (1, 15), (0, 5), (8, 24)])
def test_strides_and_alignment(kd, kind, off, pad):
    g = torch.Generator(device="cuda").manual_seed(13)
    rows, m, n = 5, 70, 200
    w = _random(kd, g, m, n, 32, True, torch.bfloat16)
    x, s = _x(g, rows, n, kind)
    ref = kd.matmul_4bit(w, x, scale=s)
    buf = torch.zeros(off + rows * (n + pad), dtype=x.dtype, device="cuda")
    xs = buf[off:].view(rows, n + pad)[:, :n]
    xs.copy_(x)
    yb = torch.full((rows, m + 9), float("nan"), device="cuda")
    kd.matmul_4bit(w, xs, scale=s, out=yb[:, :m])
    assert torch.equal(yb[:, :m], ref) and yb[:, m:].isnan().all()


def test_special_values(kd):
    """NaN and infinities of one row, or of one channel's scale, stay in that row or channel."""
    g = torch.Generator(device="cuda").manual_seed(14)
    w = _random(kd, g, 40, 300, 32, False, torch.float16)
    x, _ = _x(g, 6, 300, "f16")
    ref = kd.matmul_4bit(w, x)
    x2 = x.clone()
    x2[1, 7], x2[3, 299] = float("nan"), float("inf")
    sc = w.scales.clone()
    sc[17, 2] = float("nan")
    y = kd.matmul_4bit(kd.Weight4(w.codes, sc, n=300, group=32), x2)
    assert y[1].isnan().all() and not torch.isfinite(y[3]).any() and y[:, 17].isnan().all()
    keep = torch.ones_like(y, dtype=torch.bool)
    keep[1], keep[3], keep[:, 17] = False, False, False
    assert torch.equal(y[keep], ref[keep])


def test_large_offsets(kd):
    """Codes past 4 GB: the last channels of 540,000 x 16384."""
    m, n = 540_000, 16384
    codes = torch.empty((m, n // 8), dtype=torch.int32, device="cuda")
    codes.fill_(0x12345678)
    codes[-40:] = torch.randint(-2 ** 31, 2 ** 31, (40, n // 8), device="cuda", dtype=torch.int64).to(torch.int32)
    scales = torch.full((m, n // 32), 0.01, dtype=torch.float16, device="cuda")
    scales[-40:] *= 2 * torch.rand((40, n // 32), device="cuda").half()
    x = torch.randn((2, n), device="cuda").half()
    y = kd.matmul_4bit(kd.Weight4(codes, scales, n=n, group=32), x)
    last = kd.Weight4(codes[-40:].clone(), scales[-40:].clone(), n=n, group=32)
    _check(last, x, None, y[:, -40:])
    d = kd.dequantise_4bit(last, torch.float32)
    out = torch.empty((m, n), dtype=torch.float16, device="cuda")
    kd.dequantise_4bit(kd.Weight4(codes, scales, n=n, group=32), out=out)
    assert torch.equal(out[-40:], d.half())


def _round_up(s, dt):
    """s (fp32, not negative) rounded to the next value of dt that is not below it."""
    r = s.to(dt)
    up = (r.view(torch.int16) + 1).view(dt)      # the next one: the same sign, one further
    return torch.where(r.float() < s, up, r).float().numpy()


def _quantise_host(w, group, zeros, sdt):
    """The definition, step by step in fp32 on the host."""
    m, n = w.shape
    f = np.float32
    codes, scales, zs = np.zeros((m, n), np.int64), np.zeros((m, -(-n // group)), f), np.zeros((m, -(-n // group)), np.int64)
    for k in range(-(-n // group)):
        v = w[:, k * group:(k + 1) * group].astype(f)
        lo, hi = v.min(1), v.max(1)
        if zeros:
            lo, hi = np.minimum(lo, f(0)), np.maximum(hi, f(0))
            s = (hi - lo) / f(15)
        else:
            s = np.maximum(hi / f(7), -lo / f(8))
        s = _round_up(torch.from_numpy(s), sdt)
        ok = np.isfinite(s) & (s > 0) & np.isfinite(v).all(1)
        d = np.where(ok, s, f(1))
        z = np.where(ok, np.clip(np.rint(-lo / d), 0, 15), 0) if zeros else np.full(m, 8)
        q = np.clip(np.rint(np.where(ok[:, None], v, 0) / d[:, None]) + z[:, None], 0, 15)
        codes[:, k * group:(k + 1) * group] = np.where(ok[:, None], q, z[:, None])
        scales[:, k], zs[:, k] = s, z
    return codes, scales, zs


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("dt,sdt", [(torch.float32, torch.bfloat16), (torch.float16, torch.float16), (torch.bfloat16, torch.bfloat16)])
@pytest.mark.parametrize("m,n", [(1, 1), (5, 100), (3, 128), (20, 1000), (2, 4096)])
def test_quantise_and_dequantise_bits(kd, group, zeros, dt, sdt, m, n):
    g = torch.Generator(device="cuda").manual_seed(m + n)
    w = (torch.randn((m, n), generator=g, device="cuda") * 0.02).to(dt)
    w[0, :] = 0                      # a group of zeros
    w[-1, :] = w[-1, :].abs()        # one sign alone
    q = kd.quantise_4bit(w, group, zeros, scale_dtype=sdt)
    codes, scales, zs = _quantise_host(w.float().cpu().numpy(), group, zeros, sdt)
    assert (q.scales.float().cpu().numpy() == scales).all()
    assert (_codes(q) == codes).all()
    if zeros:
        assert (q.zeros.cpu().numpy() == zs).all()
    which = np.arange(n) // group
    dense = scales[:, which] * (codes - zs[:, which]).astype(np.float32)
    for odt in (torch.float32, torch.float16, torch.bfloat16):
        assert torch.equal(kd.dequantise_4bit(q, odt).cpu(), torch.from_numpy(dense).to(odt))


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("sdt", [torch.bfloat16, torch.float16])
def test_quantise_is_within_half_a_step(kd, zeros, sdt):
    """Many groups of every scale: no weight is further than half a step from its code's value
    (1e-5: the fp32 divisions' roundings), also where the codes end."""
    g = torch.Generator(device="cuda").manual_seed(16)
    w = torch.randn((512, 1024), generator=g, device="cuda") * 10 ** (3 * torch.rand((512, 1), generator=g, device="cuda") - 2)
    q = kd.quantise_4bit(w, 32, zeros, scale_dtype=sdt)
    step = q.scales.double().repeat_interleave(32, 1)
    assert ((kd.dequantise_4bit(q).double() - w.double()).abs() <= step * (0.5 + 1e-5)).all()


def test_quantise_special_and_strided(kd):
    w = torch.randn((4, 256), device="cuda")
    w[1, 3], w[2, 200] = float("nan"), float("inf")
    wide = torch.zeros((4, 300), device="cuda")
    wide[:, 5:261] = w
    for zeros in (False, True):
        a, b = kd.quantise_4bit(w, 64, zeros), kd.quantise_4bit(wide[:, 5:261], 64, zeros)
        assert torch.equal(a.codes, b.codes) and torch.equal(a.scales.view(torch.int16), b.scales.view(torch.int16))
        bad = ~torch.isfinite(a.scales.float())
        assert bad.nonzero().tolist() == [[1, 0], [2, 3]]
        assert torch.isfinite(a.scales[0]).all()
        out = torch.full((4, 300), 5.0, device="cuda")
        kd.dequantise_4bit(a, out=out[:, 5:261])
        assert (out[:, :5] == 5).all() and (out[:, 261:] == 5).all()
        fine = torch.isfinite(w) & ~bad.repeat_interleave(64, 1)
        step = a.scales.float().repeat_interleave(64, 1)
        # half a step, and a step at the clamped ends (the scale's rounding, 2^-9 of 8 steps)
        assert ((out[:, 5:261] - w).abs() <= step * 0.53)[fine].all()


def test_other_stream_empty_and_refusals(kd):
    g = torch.Generator(device="cuda").manual_seed(15)
    w = _random(kd, g, 64, 256, 128, False, torch.float16)
    x, _ = _x(g, 3, 256, "bf16")
    ref = kd.matmul_4bit(w, x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    a = kd.matmul_4bit(w, x, stream=s)
    with torch.cuda.stream(s):
        b = kd.matmul_4bit(w, x)
    s.synchronize()
    assert torch.equal(a, ref) and torch.equal(b, ref)
    assert kd.matmul_4bit(w, x[:0]).shape == (0, 64)
    with pytest.raises(ValueError, match="x must be"):
        kd.matmul_4bit(w, x[:, :-1])
    with pytest.raises(ValueError, match="dtype"):
        kd.matmul_4bit(w, x.float())
    with pytest.raises(ValueError, match="scale"):
        kd.matmul_4bit(w, x, scale=torch.ones(2, device="cuda"))
    with pytest.raises(ValueError, match="out"):
        kd.matmul_4bit(w, x, out=torch.empty((3, 63), device="cuda"))
    with pytest.raises(ValueError, match="contiguous"):
        kd.Weight4(w.codes.t().contiguous().t(), w.scales, n=256)
