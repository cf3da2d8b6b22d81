"""kd.matmul_4bit where its kernels do what small shapes do not make them do: rings of codes and
rows that wrap, stages of operands used again, CTAs that walk several tiles, sums of
a cluster in both of their places; against the product in 64 bits, on the GPU by blocks of
channels.  And the kernel for many rows with the outputs, strides and values of the others.

Tolerance, with A = sum_i |s (c - z) x_i| |xs|: c - z and its products with x are exact; the
tensor cores' sums of a group take at most 8 steps of 16 inputs, each of which keeps 22 bits
of its largest part: 8 * 2^-22 A.  The fp32 sums round once for each group, for each of up to 16
warps and 8 CTAs, and for the rows' scale: (groups + 25) 2^-24 A.  An output in fewer bits adds half
a unit of its type."""

import pytest
import torch

pytestmark = pytest.mark.gpu

HALF_UNIT = {torch.float32: (0.0, 2.0 ** -149), torch.float16: (torch.finfo(torch.float16).eps / 2, 2.0 ** -25),
             torch.bfloat16: (torch.finfo(torch.bfloat16).eps / 2, 2.0 ** -134)}
KINDS = {"f16": torch.float16, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}


@pytest.fixture(scope="module")
def kd():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2609_11687_gb300 import build
    build.build()
    from paper_2609_11687_gb300 import kashin
    return kashin


def _weights(kd, g, m, n, group, zeros):
    """Random codes, those past n too."""
    groups = -(-n // group)
    codes = torch.randint(-2 ** 31, 2 ** 31, (m, (n + 31) // 32 * 4), generator=g, device="cuda", dtype=torch.int64).to(torch.int32)
    scales = (torch.exp(torch.randn((groups, m), generator=g, device="cuda")) * 0.01).to(torch.bfloat16 if m % 2 else torch.float16)
    z = torch.randint(0, 16, (groups, m), generator=g, device="cuda").to(torch.uint8).t() if zeros else None
    return kd.Weight4(codes, scales.t(), z, n=n, group=group)


def _rows(g, rows, n, kind):
    x = torch.randn((rows, n), generator=g, device="cuda")
    x[:, :: max(2, n // 3)] *= 30
    if kind == "e4m3":
        s = x.abs().amax(1) / 448
        return (x / s[:, None]).to(torch.float8_e4m3fn), s
    return x.to(KINDS[kind]), None


def _check(w, x, scale, y):
    x64 = x.double() if scale is None else x.double() * scale.double()[:, None]
    which = torch.arange(w.n, device="cuda") // w.group
    shifts = torch.arange(0, 32, 4, device="cuda", dtype=torch.int32)
    rel, least = HALF_UNIT[y.dtype]
    part = 8 * 2.0 ** -22 + (w.scales.shape[1] + 25) * 2.0 ** -24
    for j in range(0, w.m, 8192):
        c = ((w.codes[j:j + 8192, :, None] >> shifts) & 15).flatten(1)[:, :w.n].double()
        c -= 8.0 if w.zeros is None else w.zeros[j:j + 8192][:, which].double()
        c *= w.scales[j:j + 8192][:, which].double()
        want, mass = x64 @ c.t(), x64.abs() @ c.abs().t()
        assert ((y[:, j:j + 8192].double() - want).abs() <= part * mass + rel * 1.01 * want.abs() + least).all()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("group,zeros", [(32, True), (64, False), (128, True), (128, False)])
@pytest.mark.parametrize("rows,m,n", [
    (17, 20011, 4096), (32, 20011, 2003), (33, 20011, 2003), (64, 20011, 4096),  # a CTA for each tile, 16 and 32 chunks
    (64, 4100, 16384), (20, 4100, 16301),                                        # clusters of eight, 16 chunks a CTA
    (64, 9000, 1500), (130, 20011, 1000)])
def test_many_chunks_of_many_rows(kd, kind, group, zeros, rows, m, n):
    g = torch.Generator(device="cuda").manual_seed(rows + n + group)
    w = _weights(kd, g, m, n, group, zeros)
    x, s = _rows(g, rows, n, kind)
    y = kd.matmul_4bit(w, x, scale=s)
    _check(w, x, s, y)
    assert torch.equal(y, kd.matmul_4bit(w, x, scale=s))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("group,zeros", [(32, False), (32, True), (64, True), (128, False), (128, True)])
@pytest.mark.parametrize("rows,m,n", [
    (1, 200_003, 500), (8, 200_003, 512), (9, 200_003, 500), (16, 200_003, 384),  # several tiles a CTA
    (1, 40_000, 16384), (8, 20_011, 16384), (9, 20_011, 16384), (16, 20_011, 16301)])  # several tiles a cluster
def test_many_tiles_of_few_rows(kd, kind, group, zeros, rows, m, n):
    g = torch.Generator(device="cuda").manual_seed(rows + n + group)
    w = _weights(kd, g, m, n, group, zeros)
    x, s = _rows(g, rows, n, kind)
    y = kd.matmul_4bit(w, x, scale=s)
    _check(w, x, s, y)
    assert torch.equal(y, kd.matmul_4bit(w, x, scale=s))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("odt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rows,m,n", [(17, 200, 700), (64, 200, 700), (64, 20011, 1000)])
def test_many_rows_16_bit_output(kd, kind, odt, rows, m, n):
    g = torch.Generator(device="cuda").manual_seed(21)
    w = _weights(kd, g, m, n, 128, False)
    x, s = _rows(g, rows, n, kind)
    y = kd.matmul_4bit(w, x, scale=s, out_dtype=odt)
    assert y.dtype == odt
    _check(w, x, s, y)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,m,n", [(20, 70, 200), (64, 300, 1000), (64, 20011, 600)])
@pytest.mark.parametrize("off,pad", [(0, 16), (1, 15), (0, 5), (8, 24)])
def test_many_rows_strides_and_alignment(kd, kind, rows, m, n, off, pad):
    g = torch.Generator(device="cuda").manual_seed(22)
    w = _weights(kd, g, m, n, 32, True)
    x, s = _rows(g, rows, n, kind)
    ref = kd.matmul_4bit(w, x, scale=s)
    buf = torch.zeros(off + rows * (n + pad), dtype=x.dtype, device="cuda")
    xs = buf[off:].view(rows, n + pad)[:, :n]
    xs.copy_(x)
    yb = torch.full((rows, m + 9), float("nan"), device="cuda")
    kd.matmul_4bit(w, xs, scale=s, out=yb[:, :m])
    assert torch.equal(yb[:, :m], ref) and yb[:, m:].isnan().all()
    _check(w, x, s, ref)


@pytest.mark.parametrize("rows,m,n", [(24, 40, 300), (64, 40, 900), (64, 20011, 900)])
def test_many_rows_special_values(kd, rows, m, n):
    """NaN and infinities of one row, or of one channel's scale, stay in that row or channel,
    also where a batch does not fill its tile."""
    g = torch.Generator(device="cuda").manual_seed(23)
    w = _weights(kd, g, m, n, 32, False)
    x, _ = _rows(g, rows, n, "f16")
    ref = kd.matmul_4bit(w, x)
    x2 = x.clone()
    x2[0, 7], x2[3, n - 1], x2[rows - 1, 0] = float("nan"), float("inf"), float("nan")
    sc = w.scales.clone()
    sc[17, 2] = float("nan")
    y = kd.matmul_4bit(kd.Weight4(w.codes, sc, n=n, group=32), x2)
    assert y[0].isnan().all() and y[rows - 1].isnan().all() and not torch.isfinite(y[3]).any() and y[:, 17].isnan().all()
    keep = torch.ones_like(y, dtype=torch.bool)
    keep[0], keep[3], keep[rows - 1], keep[:, 17] = False, False, False, False
    assert torch.equal(y[keep], ref[keep])


@pytest.mark.parametrize("group", [32, 64, 128])
def test_quantised_weights_are_within_half_a_step_and_multiply_as_expanded(kd, group):
    """The whole way: weights, codes, products, against the expanded matrix in 64 bits."""
    g = torch.Generator(device="cuda").manual_seed(24)
    dense = torch.randn((1500, 1100), generator=g, device="cuda").half() * 0.05
    for zeros in (False, True):
        w = kd.quantise_4bit(dense, group, zeros)
        step = w.scales.double().repeat_interleave(group, 1)[:, :1100]
        back = kd.dequantise_4bit(w).double()
        assert ((back - dense.double()).abs() <= step * (0.5 + 1e-5)).all()
        x, _ = _rows(g, 40, 1100, "bf16")
        _check(w, x, None, kd.matmul_4bit(w, x))
