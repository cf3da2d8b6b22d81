"""kd.rope against the formulas in 64 bits: norms, both layouts, parts of heads, strides, far
and negative positions, special values, in place, streams and graphs.

Tolerance of an output y = A (a cos - b sin): half a step of its type, and of A (|a| + |b|) what
fp32 leaves: the angle 2 pi (2^-26 + 2^-33) = 9.5e-8, sine, cosine and amplitude 3 2^-24, product
and sum 2 2^-24: 4e-7.  With a norm (sums of up to 1024 squares in chains of at most 36, of which the root
halves the error; the reciprocal root itself 4, two products) less than 44 2^-24 = 2.6e-6 more."""

import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def kd():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2609_11687_gb300 import build
    build.build()
    from paper_2609_11687_gb300 import kashin
    return kashin


def _angles(rotation, positions):
    """Whole turns taken off in integers: exact however far."""
    turns = [int(t) % 2 ** 64 for t in rotation.turns.tolist()]
    rows = [[(p * t % 2 ** 64) / 2 ** 64 * 2 * math.pi for t in turns] for p in positions.tolist()]
    return torch.tensor(rows, dtype=torch.float64, device="cuda").view(len(rows), 1, len(turns))


def _want(x, weight, rotation, positions, eps):
    """(y, the sum of sizes that its error is relative to)"""
    h = x.double()
    if weight is not None:
        h = h / (h.square().mean(2, keepdim=True) + eps).sqrt() * weight.double()
    angle, rot = _angles(rotation, positions), rotation.rot
    c, s = rotation.amplitude * angle.cos(), rotation.amplitude * angle.sin()
    y, size = h.clone(), h.abs()
    at = (slice(0, rot // 2), slice(rot // 2, rot)) if rotation.layout == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    a, b = h[..., at[0]], h[..., at[1]]
    y[..., at[0]], y[..., at[1]] = a * c - b * s, b * c + a * s
    both = rotation.amplitude * (a.abs() + b.abs())
    size[..., at[0]], size[..., at[1]] = both, both
    return y, size


def _check(got, x, weight, rotation, positions, eps=1e-6):
    want, size = _want(x, weight, rotation, positions, eps)
    half_step = torch.finfo(got.dtype).eps / 2
    least = 2.0 ** -25 if got.dtype == F16 else 0.0  # half of fp16's smallest step
    tol = half_step * want.abs() * 1.001 + (4e-7 + (0 if weight is None else 2.6e-6)) * size + least
    assert ((got.double() - want).abs() <= tol).all()


def _case(kd, tokens, hq, hk, d, rot, dt, layout, norm, far=5000, scaling=None, weight_dt=None):
    g = torch.Generator(device="cuda").manual_seed(tokens * 1000 + d)

    def randn(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    rows = randn(tokens, hq + hk + 1, d).to(dt)  # and a head of something else behind them
    weights = [(1 + 0.3 * randn(d)).to(weight_dt or dt) if norm else None for _ in range(2)]
    positions = torch.randint(0, far, (tokens,), generator=g, device="cuda")
    return rows[:, :hq], rows[:, hq:hq + hk] if hk else None, weights, positions, kd.Rotation(rot, layout=layout, scaling=scaling)


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dt", [F16, BF16, F32])
@pytest.mark.parametrize("tokens,hq,hk,d,rot", [
    (1, 32, 8, 128, 128), (5, 3, 1, 80, 32), (7, 2, 2, 64, 64), (3, 5, 0, 96, 96), (2, 1, 1, 2, 2), (4, 3, 3, 257, 256),
    (2, 2, 1, 1024, 1024), (300, 4, 2, 128, 64), (33, 1, 1, 72, 16), (2000, 7, 1, 64, 64), (6, 3, 2, 50, 30)])
def test_rope(kd, tokens, hq, hk, d, rot, dt, layout, norm):
    q, k, weights, positions, rotation = _case(kd, tokens, hq, hk, d, rot, dt, layout, norm)
    yq, yk = kd.rope(q, k, positions, rotation, weights[0], weights[1] if hk else None)
    _check(yq, q, weights[0], rotation, positions)
    if hk:
        _check(yk, k, weights[1], rotation, positions)
    else:
        assert yk is None


def test_weights_in_fp32_and_of_one_side(kd):
    q, k, weights, positions, rotation = _case(kd, 9, 4, 2, 128, 128, BF16, "half", True, weight_dt=F32)
    yq, yk = kd.rope(q, k, positions, rotation, None, weights[1])
    _check(yq, q, None, rotation, positions)
    _check(yk, k, weights[1], rotation, positions)
    yq, yk = kd.rope(q, k, positions, rotation, weights[0], None, eps=0.5)
    _check(yq, q, weights[0], rotation, positions, eps=0.5)
    _check(yk, k, None, rotation, positions)


@pytest.mark.parametrize("kind", ["linear", "bands", "ramp"])
def test_far_and_negative_positions(kd, kind):
    """Against the integers, whose only error is the table's; and the same frequencies times
    positions in 64-bit floating point, which lose 2^-52 of the angle each (table and product)."""
    q, k, _, _, rotation = _case(kd, 8, 2, 1, 128, 128, F32, "half", False, scaling=kd.Scaling(kind, 8.0, 4096))
    positions = torch.tensor([0, 1, -1, 2 ** 20 + 1, -(2 ** 31) - 7, 2 ** 40 + 3, -(2 ** 62), 2 ** 63 - 1], device="cuda")
    yq, yk = kd.rope(q, k, positions, rotation)
    _check(yq, q, None, rotation, positions)
    _check(yk, k, None, rotation, positions)
    near = positions[:5]
    angle = near.double()[:, None] * torch.from_numpy(rotation.frequencies).cuda()
    a, b = q[:5].double().chunk(2, 2)
    want = torch.cat((a * angle.cos()[:, None] - b * angle.sin()[:, None], b * angle.cos()[:, None] + a * angle.sin()[:, None]), 2)
    size = (a.abs() + b.abs()).repeat(1, 1, 2)
    lost = 2.0 ** -51 * near.abs().double()[:, None, None]
    assert ((yq[:5].double() - rotation.amplitude * want).abs() <= 1.5 * size * (4.6e-7 + lost)).all()


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("d,rot", [(128, 128), (80, 32), (66, 30)])
def test_in_place(kd, d, rot, layout):
    q, k, weights, positions, rotation = _case(kd, 50, 6, 2, d, rot, F16, layout, True)
    base = q._base if q._base is not None else q
    behind = base[:, -1].clone()
    want = kd.rope(q, k, positions, rotation, *weights)
    got = kd.rope(q, k, positions, rotation, *weights, out=(q, k))
    assert got[0] is q and got[1] is k
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(base[:, -1], behind)


def test_outputs_with_gaps_and_head_major(kd):
    """What lies between the written heads stays, and the bits go by neither layout nor batch."""
    q, k, weights, positions, rotation = _case(kd, 21, 4, 2, 64, 64, BF16, "half", True)
    want = kd.rope(q, k, positions, rotation, *weights)
    wide = torch.full((21, 4, 100), 7.0, dtype=BF16, device="cuda")
    major = torch.full((2, 21, 64), 7.0, dtype=BF16, device="cuda")
    kd.rope(q, k, positions, rotation, *weights, out=(wide[..., 3:67], major.transpose(0, 1)))
    assert torch.equal(wide[..., 3:67], want[0]) and torch.equal(major.transpose(0, 1), want[1])
    assert (wide[..., :3] == 7).all() and (wide[..., 67:] == 7).all()
    one = kd.rope(q[5:6], k[5:6], positions[5:6], rotation, *weights)
    assert torch.equal(one[0], want[0][5:6]) and torch.equal(one[1], want[1][5:6])


def test_broadcast_heads(kd):
    """One head shown as several (stride 0) is read as such."""
    q, _, _, positions, rotation = _case(kd, 5, 1, 1, 64, 64, F16, "half", False)
    y, _ = kd.rope(q.expand(5, 3, 64), None, positions, rotation)
    one, _ = kd.rope(q, None, positions, rotation)
    assert torch.equal(y, one.expand(5, 3, 64))


@pytest.mark.parametrize("d", [64, 50])
def test_special_values_stay_where_they_are(kd, d):
    q, k, weights, positions, rotation = _case(kd, 4, 3, 1, d, 32, F16, "half", True)
    clean = kd.rope(q, k, positions, rotation)[0], kd.rope(q, k, positions, rotation, *weights)[0]
    q[1, 2, 5], q[2, 0, 40], q[3, 1, 0] = math.inf, math.nan, -math.inf
    y = kd.rope(q, k, positions, rotation)[0]
    touched = torch.zeros(q.shape, dtype=torch.bool, device="cuda")
    for at in ((1, 2, 5), (1, 2, 21), (2, 0, 40), (3, 1, 0), (3, 1, 16)):
        touched[at] = True
    assert torch.equal(y[~touched], clean[0][~touched]) and not torch.isfinite(y[touched]).any()
    y = kd.rope(q, k, positions, rotation, *weights)[0]
    touched = torch.zeros(q.shape[:2], dtype=torch.bool, device="cuda")
    touched[1, 2] = touched[2, 0] = touched[3, 1] = True
    assert torch.equal(y[~touched], clean[1][~touched]) and y[touched].isnan().all()


def test_nothing_to_do(kd):
    rotation = kd.Rotation(64)
    q = torch.empty((0, 4, 64), dtype=F16, device="cuda")
    positions = torch.empty(0, dtype=torch.int64, device="cuda")
    assert kd.rope(q, None, positions, rotation)[0].shape == (0, 4, 64)
    q = torch.empty((3, 0, 64), dtype=F16, device="cuda")
    assert kd.rope(q, None, torch.arange(3, device="cuda"), rotation)[0].shape == (3, 0, 64)


def test_stream_and_graph(kd):
    q, k, weights, positions, rotation = _case(kd, 40, 4, 2, 128, 128, BF16, "half", True)
    want = kd.rope(q, k, positions, rotation, *weights)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = kd.rope(q, k, positions, rotation, *weights, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = kd.rope(q, k, positions, rotation, *weights)
    q.copy_(torch.randn_like(q))
    positions.add_(17)
    graph.replay()
    torch.cuda.synchronize()
    want = kd.rope(q, k, positions, rotation, *weights)
    assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])


def test_turns_of_known_angles(kd):
    """A quarter, an eighth and ten and a half turns."""
    r = kd.Rotation(6, frequencies=np.array([math.pi / 2, -math.pi / 4, 21 * math.pi]))
    got = r.turns.cpu().numpy().view(np.uint64) / 2.0 ** 64
    assert np.allclose(got, [0.25, 0.875, 0.5], rtol=0, atol=21 * 2.0 ** -52)
