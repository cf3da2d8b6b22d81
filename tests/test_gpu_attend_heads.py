"""The attention step's queries, keys and values against 64 bits from its weights: which rows of the projection they are,
whose norm's weight each takes, its eps, the rotation's positions."""

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
@pytest.mark.parametrize("eps", [1e-5, 0.5])
@pytest.mark.parametrize("hidden,heads,kv_heads,d,rot,tokens,normed", [(256, 4, 2, 64, 64, 1, True), (256, 4, 2, 64, 64, 40, True),
                                                                       (384, 3, 3, 128, 32, 7, True), (320, 8, 1, 80, 80, 70, True),
                                                                       (256, 4, 2, 64, 64, 9, False)])
def test_queries_keys_and_values(kd, hidden, heads, kv_heads, d, rot, tokens, normed, eps, dt):
    """From the 8-bit rows of the input norm on (its own test has them).  A product x is off by half a step of its type and 1e-5 of
    its terms' sizes (fp32 sums); a norm's factor r by the share of its head that these are, in the root of squares; a turned
    channel by both of its pair's errors and 2^-20 (angles to 2^-25 turns, fp32); the result by half a step more."""
    from paper_2609_11687_gb300.attend import AttentionStep
    g = torch.Generator(device="cuda").manual_seed(hidden + d + tokens)

    def randn(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    qkv = (randn((heads + 2 * kv_heads) * d, hidden) * hidden ** -0.5).to(dt)
    qkv *= (0.25 + torch.arange((heads + 2 * kv_heads) * d, device="cuda") % 7 / 7)[:, None].to(dt)
    out = (randn(hidden, heads * d) * (heads * d) ** -0.5).to(dt)
    norm, q_norm, k_norm = (1 + 0.1 * randn(hidden)).to(dt), (1 + 0.1 * randn(d)).to(dt), (3 + 0.5 * randn(d)).to(dt)
    weights = (q_norm, k_norm) if normed else ()
    step = AttentionStep(norm, qkv, out, kd.new_cache_4bit(4, kv_heads, d, 16, 64), kd.Rotation(rot), *weights, eps=eps)
    x, residual = randn(tokens, hidden).to(dt), randn(tokens, hidden).to(dt)
    positions = torch.randint(0, 5000, (tokens,), generator=g, device="cuda")
    q, k, v, new = step.heads_of(x, positions, residual)
    total = (x.float() + residual.float()).to(dt)
    assert torch.equal(new, total)
    rows = kd.rmsnorm(x, norm, eps, residual=residual)
    dense = kd.dequantise_4bit(step.qkv).double()
    a = rows.q.double() * rows.scale.double()[:, None]
    # the input norm's own formula, to the 8-bit rows' half step, that of the sum, and half of the smallest 8-bit number
    h = total.double() * (total.double().square().mean(1, keepdim=True) + eps).rsqrt() * norm.double()
    half = torch.finfo(dt).eps / 2
    assert ((a - h).abs() <= (2.0 ** -4 + 2 * half) * 1.01 * h.abs() + 2.0 ** -9 * rows.scale.double()[:, None]).all()
    p = (a @ dense.t()).view(tokens, heads + 2 * kv_heads, d)
    off = half * p.abs() + 1e-5 * (a.abs() @ dense.abs().t()).view_as(p) + 2.0 ** -25
    f = 10000.0 ** (-2.0 * torch.arange(rot // 2, dtype=torch.float64, device="cuda") / rot)
    cos, sin = torch.cos(positions[:, None, None] * f), torch.sin(positions[:, None, None] * f)
    for got, at, weight in ((q, slice(0, heads), q_norm), (k, slice(heads, heads + kv_heads), k_norm)):
        y, e = p[:, at], off[:, at]
        if normed:
            r = (y.square().mean(2, keepdim=True) + eps).rsqrt()
            share = e.norm(dim=2, keepdim=True) / y.norm(dim=2, keepdim=True)
            e = (e + y.abs() * share) * (1 + share) * r * weight.double().abs()
            y = y * r * weight.double()
        want, tol = y.clone(), e.clone()
        u, w = y[..., :rot // 2], y[..., rot // 2:rot]
        want[..., :rot // 2], want[..., rot // 2:rot] = u * cos - w * sin, w * cos + u * sin
        both = e[..., :rot // 2] + e[..., rot // 2:rot] + 2.0 ** -20 * (u.abs() + w.abs())
        tol[..., :rot // 2], tol[..., rot // 2:rot] = both, both
        assert ((got.double() - want).abs() <= tol + half * 1.01 * want.abs() + 2.0 ** -20 * want.abs() + 2.0 ** -25).all()
    values = slice(heads + kv_heads, heads + 2 * kv_heads)
    assert ((v.double() - p[:, values]).abs() <= off[:, values]).all()
