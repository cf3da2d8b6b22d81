"""kd.attention_4bit where steps of values differ by many powers of two: large and infinite ones that a row does not see leave
its bits, and ones that it sees leave the digits of what weighs more and of other groups of channels.

Tolerance of an output, with weights w = exp(x - max) / z, values v and middles v0 = low + 8 step:
  half a step of its type, relative to it;
  2^-11 sum w |v - v0|: weights times steps are rounded to fp16 (half a step is 2^-11 of a value at most), codes count from 8;
  2^-12 S / z: sums of sixteen products on the tensor cores drop what lies that far below the largest (as measured);
  (2 delta + 2^-20) sum w (|v| + |v0| + 8 step): delta is the largest error of a score of the row, fp32 sums of d products in steps of
    sixteen (each step and each of up to 40 other operations 2^-23 of the sum of sizes), of the positions within e^100 of the row's
    heaviest: others weigh nothing in either form (up to 2^18 of them e^-80);
  n 2^-27 S / z + n 2^-51 / z: S is the largest exp(x - max) step of the row and the group.  Products of weights and steps are in units
    that bring S to 2^5 at least (or are as small as they get, 2^-29), of which fp16's smallest numbers are off by 2^-25, times eight;
  2^-25, half of fp16's smallest step."""

import math

import pytest
import torch

from test_gpu_attention4 import BF16, F16, NONE, Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kd():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2609_11687_gb300 import build
    build.build()
    from paper_2609_11687_gb300 import kashin
    return kashin


def _place(c, s, pos):
    return c.seqs.table[s, pos // c.page].long(), slice(None), pos % c.page


SIZES = [4000.0, 60000.0, math.inf, -math.inf]


@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("hq,hk,d,group,room", [(4, 1, 128, 64, 0), (1, 1, 64, 32, 0), (2, 2, 128, 128, 0), (8, 1, 128, 32, 0), (3, 1, 256, 64, 0),
                                                (4, 1, 128, 64, 200000), (1, 1, 128, 64, 200000), (6, 2, 80, 32, 200000), (2, 1, 200, 128, 200000)])
def test_large_steps_that_a_row_does_not_see(kd, hq, hk, d, group, room, size):
    """A large or infinite step, or lowest value, of the last drafted token's value, and of the first position of the first
    row's window: the rows that do not see it keep their bits."""
    for which in (0, 1):  # step, low
        c = Case(kd, [700, 45], [4, 2], hq, hk, d, group=group, steps=2.0 ** -9, room=room)
        clean = c.check(kd)
        for s, length in enumerate(c.lengths):
            c.cache.v_scales[(*_place(c, s, length - 1), slice(None), which)] = abs(size) if which == 0 else size
        out, lse = c.run(kd)
        others, last = [0, 1, 2, 4], [3, 5]
        assert torch.equal(out[others], clean[0][others]) and torch.equal(lse, clean[1])
        assert not torch.equal(out[last], clean[0][last])
    for window in (1, 20, 300):
        c = Case(kd, [700, 45], [4, 2], hq, hk, d, group=group, steps=2.0 ** -9, room=room)
        clean = c.check(kd, window=window)
        for s, (length, n) in enumerate(zip(c.lengths, c.counts)):
            if length - n + 1 - window >= 0:
                c.cache.v_scales[(*_place(c, s, length - n + 1 - window), slice(None), 0)] = abs(size)
        out, lse = c.run(kd, window=window)
        assert torch.equal(out[1:4], clean[0][1:4]) and torch.equal(out[5], clean[0][5]) and torch.equal(lse, clean[1])
        assert not torch.equal(out[0], clean[0][0])


def _check(kd, c):
    out, lse = c.run(kd)
    eps, scale, group = torch.finfo(c.q.dtype).eps / 2, c.d ** -0.5, torch.arange(c.d, device="cuda") // c.group
    for s, (n, length) in enumerate(zip(c.counts, c.lengths)):
        rows = slice(int(c.starts[s]), int(c.starts[s + 1]))
        (k, k0, kstep), (v, v0, vstep) = c.dense("k", s), c.dense("v", s)
        v0 = v0 + 0.5 * vstep
        qs = c.q[rows].double().view(n, c.hk, c.hq // c.hk, c.d)
        seen = (torch.arange(length, device="cuda") <= torch.arange(length - n, length, device="cuda")[:, None])[:, None, None]
        x = (torch.einsum("nhgd,lhd->nhgl", qs, k) * scale).masked_fill(~seen, NONE)
        e = (x - x.amax(-1, keepdim=True)).exp()
        z = e.sum(-1, keepdim=True)
        size = torch.einsum("nhgd,lhd->nhgl", qs.abs(), (k - k0 + 7.5 * kstep).abs() + (k0 - 7.5 * kstep).abs()) * scale
        delta = torch.where(x > x.amax(-1, keepdim=True) - 100, size, torch.zeros_like(size)).amax(-1, keepdim=True) * (c.d / 16 + 40) * 2.0 ** -23
        want = torch.einsum("nhgl,lhd->nhgd", e / z, v)
        most = torch.stack([(e.permute(3, 1, 0, 2) * vstep[:, :, None, None, i * c.group]).amax(0) for i in range(int(group[-1]) + 1)], -1).permute(1, 0, 2, 3)
        tol = eps * want.abs() * 1.001 + 2.0 ** -11 * torch.einsum("nhgl,lhd->nhgd", e / z, (v - v0).abs()) \
            + (2 * delta + 2.0 ** -20) * torch.einsum("nhgl,lhd->nhgd", e / z, v.abs() + v0.abs() + 8 * vstep) \
            + ((length * 2.0 ** -27 + 2.0 ** -12) * most[..., group] + length * 2.0 ** -51) / z + 2.0 ** -25
        off = (out[rows].double() - want.reshape(n, c.hq, c.d)).abs() / tol.reshape(n, c.hq, c.d)
        assert off.max() <= 1, float(off.max())


@pytest.mark.parametrize("d,group,hq,hk,room", [(128, 64, 4, 1, 0), (128, 32, 8, 1, 0), (64, 32, 3, 1, 0), (256, 64, 8, 2, 0), (128, 64, 4, 1, 200000),
                                                (96, 32, 8, 1, 200000), (256, 128, 2, 1, 200000)])
@pytest.mark.parametrize("dt", [F16, BF16])
@pytest.mark.parametrize("at", [0, 399, "all along"])
def test_large_steps_of_no_weight(kd, d, group, hq, hk, room, dt, at):
    """Positions with steps 2^24 times the others' whose keys lie so far from the queries that they weigh nothing, seen
    by all rows: at the start, at the end and between the others."""
    c = Case(kd, [400, 77], [1, 1], hq, hk, d, group=group, dt=dt, steps=2.0 ** -9, room=room)
    # all queries lean to one side, and so do the keys of these positions, the other way
    c.q = (c.q.float() + 1).to(dt)
    for s, length in enumerate(c.lengths):
        for pos in (range(0, length, 37) if at == "all along" else [min(at, length - 1)]):
            c.cache.v_scales[(*_place(c, s, pos), slice(None), 0)] = 60000.0
            c.cache.v_scales[(*_place(c, s, pos), slice(None), 1)] = 0.0
            c.cache.k_scales[(*_place(c, s, pos), slice(None), 0)] = 0.0
            c.cache.k_scales[(*_place(c, s, pos), slice(None), 1)] = -1000.0
    _check(kd, c)


@pytest.mark.parametrize("hq,hk,room", [(4, 1, 0), (8, 1, 0), (8, 1, 200000), (2, 1, 200000)])
@pytest.mark.parametrize("d,group", [(128, 64), (128, 32), (256, 64), (80, 32)])
def test_groups_of_unlike_steps(kd, hq, hk, room, d, group):
    """Groups of channels whose steps lie 2^23 apart, in either order."""
    for order in (1, -1):
        c = Case(kd, [300, 40], [2, 1], hq, hk, d, group=group, steps=2.0 ** -9, room=room)
        n = c.cache.v_scales.shape[3]
        power = 2.0 ** (23.0 * torch.arange(n, device="cuda") / max(n - 1, 1))
        power = power if order == 1 else power.flip(0)
        c.cache.v_scales.copy_((c.cache.v_scales.float() * power[:, None]).clamp(-60000, 60000))
        c.check(kd)
        _check(kd, c)


def test_scores_that_rise_as_steps_fall(kd):
    """Each position outweighs all before it and has a smaller step: the units follow at every move of the maximum."""
    for d, group, heads in ((128, 64, 8), (128, 32, 3), (256, 64, 2)):
        for length in (40, 300, 1500):
            c = Case(kd, [length], [1], heads, 1, d, group=group)
            c.q = torch.ones_like(c.q)
            at = torch.arange(length, device="cuda")
            page, place = c.seqs.table[0].long()[at // c.page], at % c.page
            turn = at.float() / length
            c.cache.k_scales[page, :, place, :, 0] = 0
            c.cache.k_scales[page, :, place, :, 1] = (turn * 150 / d ** 0.5).half()[:, None, None]
            c.cache.v_scales[page, :, place, :, 0] = torch.exp2(14 - 24 * turn).half()[:, None, None]
            c.cache.v_scales[page, :, place, :, 1] = 0
            _check(kd, c)
