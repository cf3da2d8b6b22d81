"""kd.attention_4bit against softmax(scale q k^T) v in 64 bits over the values that the cache holds:
types, sizes, masks, pages, splits, special values where a row looks and where it does not.

Tolerance of an output with weights w (of sum 1), values v and middles v0 = low + 7.5 step:
  half a step of its type, relative to it;
  2^-11 sum w |v - v0|: weights times steps are rounded to fp16;
  (2 delta + 2^-20) sum w |v|: delta is the largest error of a score of the row, fp32 sums of d products in
    steps of sixteen (each step and each of up to 40 other operations 2^-23 of the sum of sizes);
  n 2^-27 max step / sum exp(x - max): n weights that may fall below fp16's normal range;
  2^-25, half of fp16's smallest step.
lse: delta, and 2^-20 of its size (at least 1)."""

import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
NONE = -math.inf


@pytest.fixture(scope="module")
def kd():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2609_11687_gb300 import build
    build.build()
    from paper_2609_11687_gb300 import kashin
    return kashin


class Case:
    def __init__(self, kd, lengths, counts, hq, hk, d, page=16, group=64, dt=F16, uniform=False, spare=0, seed=0, longest=None, steps=1.0, room=0):
        g = torch.Generator(device="cuda").manual_seed(seed + 7 * d + len(lengths))
        self.lengths, self.counts, self.hq, self.hk, self.d, self.page, self.group = lengths, counts, hq, hk, d, page, group
        seqs, wide = len(lengths), max(1, -(-max(max(lengths), 1) // page))
        pages = seqs * wide + 1
        self.cache = kd.new_cache_4bit(pages, hk, d, page, group)
        for codes, scales in ((self.cache.k_codes, self.cache.k_scales), (self.cache.v_codes, self.cache.v_scales)):
            c = torch.randint(0, 16, (*codes.shape[:3], codes.shape[3] * 8), generator=g, device="cuda")
            c[..., d:] = 0
            packed = (c.view(*codes.shape, 8) << torch.arange(0, 32, 4, device="cuda")).sum(-1)
            codes.copy_(torch.where(packed >= 2 ** 31, packed - 2 ** 32, packed).int())
            step = torch.exp(0.3 * torch.randn(scales.shape[:-1], generator=g, device="cuda")) * 0.2 * steps
            scales[..., 0] = step
            scales[..., 1] = step * (torch.randn(step.shape, generator=g, device="cuda") - 7.5)
        table = torch.randperm(pages, generator=g, device="cuda")[:seqs * wide].view(seqs, wide).int()
        if room:  # a table for sequences of that length, of which no page is there yet
            table = torch.cat((table, torch.full((seqs, room // page - wide), -1, dtype=torch.int32, device="cuda")), 1)
            longest = room
        self.starts = np.concatenate(([0], np.cumsum(counts))).astype(int)
        most = max(counts)
        i32 = dict(dtype=torch.int32, device="cuda")
        self.seqs = kd.Sequences(table, torch.tensor(lengths, **i32), None if uniform else torch.tensor(self.starts.tolist(), **i32),
                                 most=most, longest=max(lengths) if longest is None else longest)
        tokens = int(self.starts[-1]) + spare
        self.q = (torch.randn((tokens, hq, d), generator=g, device="cuda") * 1.5 * math.sqrt(64 / max(d, 16))).to(dt)

    def dense(self, which, s):
        """(places, hk, d) values of a sequence in 64 bits, and their middles and steps"""
        codes, scales = (self.cache.k_codes, self.cache.k_scales) if which == "k" else (self.cache.v_codes, self.cache.v_scales)
        at = torch.arange(self.lengths[s], device="cuda")
        pg, place = self.seqs.table[s].long()[at // self.page], at % self.page
        w, sc = codes[pg, :, place].long() & 0xFFFFFFFF, scales[pg, :, place].double()
        ch = torch.arange(self.d, device="cuda")
        c = (w[..., ch // 8] >> (4 * (ch % 8)) & 15).double()
        step, low = sc[..., ch // self.group, 0], sc[..., ch // self.group, 1]
        return low + step * c, low + 7.5 * step, step

    def want(self, scale=None, causal=True, window=0):
        """out, lse, and the tolerance of each"""
        scale = self.d ** -0.5 if scale is None else scale
        q, G = self.q.double(), self.hq // self.hk
        out, lse = torch.zeros_like(q), torch.full(q.shape[:2], NONE, dtype=torch.float64, device="cuda")
        tol, ltol = torch.zeros_like(q), torch.zeros_like(lse)
        eps = torch.finfo(self.q.dtype).eps / 2
        for s, (n, length) in enumerate(zip(self.counts, self.lengths)):
            if n == 0 or length == 0:
                continue
            rows = slice(int(self.starts[s]), int(self.starts[s + 1]))
            k, k0, kstep = self.dense("k", s)
            v, v0, vstep = self.dense("v", s)
            pos, own = torch.arange(length, device="cuda"), torch.arange(length - n, length, device="cuda")[:, None]
            seen = torch.ones((n, length), dtype=torch.bool, device="cuda")
            if causal:
                seen = pos <= own
                if window:
                    seen &= pos > own - window
            qs = q[rows].view(n, self.hk, G, self.d)
            x = torch.einsum("nhgd,lhd->nhgl", qs, k) * scale
            x = torch.where(seen[:, None, None], x, torch.full_like(x, NONE))
            top = x.amax(-1, keepdim=True)
            none = top == NONE
            e = (x - torch.where(none, torch.zeros_like(top), top)).exp()
            z = e.sum(-1, keepdim=True)
            w = torch.where(none, torch.zeros_like(e), e / z)
            # sizes of a score's terms: code times step, and low
            size = torch.einsum("nhgd,lhd->nhgl", qs.abs(), (k - k0 + 7.5 * kstep).abs() + (k0 - 7.5 * kstep).abs()) * abs(scale)
            delta = torch.where(seen[:, None, None], size, torch.zeros_like(size)).amax(-1, keepdim=True) * (self.d / 16 + 40) * 2.0 ** -23
            o = torch.einsum("nhgl,lhd->nhgd", w, v)
            t = eps * o.abs() * 1.001 + 2.0 ** -11 * torch.einsum("nhgl,lhd->nhgd", w, (v - v0).abs()) \
                + (2 * delta + 2.0 ** -20) * torch.einsum("nhgl,lhd->nhgd", w, v.abs() + v0.abs() + 7.5 * vstep) \
                + seen.sum(1)[:, None, None, None] * 2.0 ** -27 * vstep.amax() / torch.where(none, torch.ones_like(z), z) + 2.0 ** -25
            out[rows], tol[rows] = o.reshape(n, self.hq, self.d), t.reshape(n, self.hq, self.d)
            ls = torch.where(none, top, top + z.log())[..., 0]
            lse[rows] = ls.reshape(n, self.hq)
            ltol[rows] = (delta[..., 0] + 2.0 ** -20 * torch.where(none[..., 0], torch.zeros_like(ls), ls).abs().clamp(min=1)).reshape(n, self.hq)
        return out, lse, tol, ltol

    def run(self, kd, **k):
        lse = torch.full(self.q.shape[:2], 77.0, dtype=F32, device="cuda")
        out = torch.full_like(self.q, 7.0)
        got = kd.attention_4bit(self.cache, self.q, self.seqs, out=out, lse=lse, **k)
        assert got is out
        return out, lse

    def check(self, kd, **k):
        out, lse = self.run(kd, **k)
        n = int(self.starts[-1])
        assert (out[n:] == 7).all() and (lse[n:] == 77).all()  # rows of no sequence
        k.pop("workspace", None)
        want, wlse, tol, ltol = self.want(**k)
        off = (out.double() - want).abs()[:n]
        assert (off <= tol[:n]).all(), float((off / tol[:n]).max())
        none = wlse[:n] == NONE
        assert torch.equal(none, lse[:n] == NONE)
        assert ((lse.double() - wlse).abs()[:n][~none] <= ltol[:n][~none]).all()
        return out, lse


@pytest.mark.parametrize("dt", [F16, BF16])
@pytest.mark.parametrize("d,group", [(128, 32), (128, 64), (128, 128), (64, 32), (64, 64), (64, 128), (32, 32), (32, 128), (96, 32),
                                     (96, 64), (96, 128), (192, 64), (160, 32), (256, 32), (256, 64), (256, 128), (80, 32), (37, 64),
                                     (1, 32), (200, 128), (100, 32), (250, 64), (129, 128)])
def test_heads_and_groups(kd, d, group, dt):
    Case(kd, [1, 17, 100, 0, 333], [1, 1, 1, 1, 1], 4, 2, d, group=group, dt=dt).check(kd)
    Case(kd, [1, 17, 100, 0, 333], [1, 3, 2, 1, 5], 4, 2, d, group=group, dt=dt).check(kd)


@pytest.mark.parametrize("d,group", [(128, 32), (128, 64), (128, 128), (64, 32), (64, 64), (32, 32), (96, 32), (96, 64), (96, 128),
                                     (160, 32), (160, 64), (160, 128), (192, 32), (192, 64), (192, 128), (224, 32), (224, 64), (224, 128),
                                     (256, 32), (256, 64), (256, 128)])
@pytest.mark.parametrize("drafted", [0, 1])
def test_equal_shares(kd, d, group, drafted):
    """Lengths that may be long (the host knows the table's room only): equal shares of all positions for
    every CTA, of which one here has several items, another a part of one."""
    rng = np.random.RandomState(d)
    lengths = rng.randint(0, 900, 40).tolist() + [0, 5000, 1, 3]
    c = Case(kd, lengths, [1] * 20 + [1 + drafted, 0] * 12, 6, 2, d, group=group, dt=BF16, spare=1, room=100000)
    assert kd.attention_4bit_workspace(c.cache, c.seqs, 6) > 0
    first = c.check(kd)
    again = c.run(kd)
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
    c.check(kd, window=300)
    c.check(kd, causal=False)


@pytest.mark.parametrize("hq,hk,most", [(1, 1, 1), (8, 1, 1), (9, 1, 1), (16, 1, 1), (17, 1, 1), (32, 8, 1), (32, 32, 1), (40, 8, 1), (7, 7, 3),
                                        (6, 2, 4), (4, 4, 9), (10, 2, 7), (8, 1, 33), (64, 1, 2)])
@pytest.mark.parametrize("d", [64, 128, 160])
def test_heads_that_share_and_drafted_tokens(kd, hq, hk, most, d):
    rng = np.random.RandomState(hq + most)
    counts = [most, 1, 0, min(2, most), max(1, most // 2)]
    lengths = [200, 1, 50, 15, 64 + int(rng.randint(0, 300))]
    Case(kd, lengths, counts, hq, hk, d, dt=BF16, spare=3).check(kd)


@pytest.mark.parametrize("length", [1, 2, 15, 16, 17, 127, 128, 129, 255, 256, 257, 1000, 4096, 4097, 5000])
def test_lengths(kd, length):
    Case(kd, [length], [1], 8, 2, 64, uniform=True).check(kd)
    Case(kd, [length, length], [min(3, length)] * 2, 4, 2, 128, page=64, uniform=True, dt=BF16).check(kd)


@pytest.mark.parametrize("page", [16, 32, 48, 128, 1024])
@pytest.mark.parametrize("window", [0, 1, 5, 16, 17, 100, 10000])
def test_windows_and_pages(kd, page, window):
    Case(kd, [700, 3, 0, 129], [4, 2, 1, 1], 6, 2, 64, page=page, group=32).check(kd, window=window)


def test_without_causal_and_scales(kd):
    c = Case(kd, [300, 20, 1], [5, 3, 1], 4, 2, 128)
    c.check(kd, causal=False)
    c.check(kd, scale=0.0)
    c.check(kd, scale=-0.05)
    c.check(kd, scale=1.0)


def test_positions_below_zero(kd):
    """Sequences shorter than their rows of the call: the first rows see nothing."""
    c = Case(kd, [2, 5], [4, 5], 4, 2, 64)
    out, lse = c.run(kd)
    assert (out[:2] == 0).all() and (lse[:2] == NONE).all() and torch.isfinite(lse[2:]).all()
    c.lengths, c.counts, c.starts = [2, 5], [2, 5], np.array([2, 4, 9])
    want, wlse, tol, ltol = c.want()
    assert ((out.double() - want).abs()[2:] <= tol[2:]).all() and ((lse.double() - wlse).abs()[2:] <= ltol[2:]).all()
    out, lse = c.run(kd, causal=False)  # all of them see all
    assert torch.isfinite(lse).all()


@pytest.mark.parametrize("lengths,hq,hk,d,group", [([40000], 8, 2, 128, 64), ([70001], 4, 1, 64, 32), ([20000, 1, 0, 7777], 8, 1, 128, 128),
                                                   ([9000] * 3, 40, 1, 96, 64), ([30000], 2, 2, 256, 128),
                                                           ([25000] * 3, 40, 1, 96, 64), ([3000] * 90, 8, 4, 64, 64)])
def test_long_sequences_in_shares(kd, lengths, hq, hk, d, group):
    c = Case(kd, lengths, [1] * len(lengths), hq, hk, d, page=64, group=group, dt=BF16)
    if lengths in ([40000], [25000] * 3):  # equal shares for all CTAs, joined by a second launch
        assert kd.attention_4bit_workspace(c.cache, c.seqs, hq) > 0
    first = c.check(kd)
    again = c.run(kd)
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
    c.check(kd, window=5000)


def test_many_sequences(kd):
    rng = np.random.RandomState(3)
    Case(kd, rng.randint(0, 60, 700).tolist(), [1] * 700, 8, 2, 64, uniform=True).check(kd)
    Case(kd, rng.randint(5, 3000, 60).tolist(), rng.randint(0, 4, 60).tolist(), 8, 4, 128, page=32, dt=BF16, spare=2).check(kd)


def test_a_hint_that_is_wrong(kd):
    """Lengths past `longest` are taken in longer shares; without it the table's room is the hint."""
    for longest in (0, 1, 1000, None):
        c = Case(kd, [20000, 300], [2, 2], 8, 2, 64, page=64, longest=longest)
        if longest is None:
            c.seqs = kd.Sequences(c.seqs.table, c.seqs.lengths, c.seqs.starts, most=2)
        c.check(kd)


def _spoil(c, keep_k, keep_v):
    """NaN and infinities wherever `keep` (pages, hk, page) does not hold."""
    for scales, keep in ((c.cache.k_scales, keep_k), (c.cache.v_scales, keep_v)):
        bad = torch.tensor([math.nan, math.inf, NONE], device="cuda").half()[torch.arange(scales.numel(), device="cuda") % 3].view(scales.shape)
        scales.copy_(torch.where(keep[..., None, None], scales, bad))


def test_what_a_row_does_not_see_does_not_touch_it(kd):
    """Places behind the sequences' ends, before their windows and in no sequence hold NaN and
    infinities, pages there have numbers that do not exist: the same bits."""
    for window, d, group in ((0, 64, 32), (40, 128, 64), (40, 80, 128)):
        c = Case(kd, [100, 33, 0, 250], [3, 1, 2, 2], 6, 2, d, group=group)
        clean = c.check(kd, window=window)
        keep = torch.zeros(c.cache.k_codes.shape[:3], dtype=torch.bool, device="cuda")
        for s, (n, length) in enumerate(zip(c.counts, c.lengths)):
            lo = max(0, length - n + 1 - window) if window else 0
            for pos in range(lo, length):
                keep[c.seqs.table[s, pos // 16], :, pos % 16] = True
            for pg in range(c.seqs.table.shape[1]):
                if 16 * pg >= length or 16 * pg + 16 <= lo:
                    c.seqs.table[s, pg] = (-1, 2 ** 31 - 1, -2 ** 31, c.cache.pages)[pg % 4]
        _spoil(c, keep, keep)
        got = c.run(kd, window=window)
        assert torch.equal(got[0], clean[0]) and torch.equal(got[1], clean[1])


def test_drafted_tokens_do_not_see_what_comes_after(kd):
    """NaN in the last token's key and value: the rows before it keep their bits."""
    for spoiled in ("k", "v"):
        c = Case(kd, [80, 21], [5, 2], 4, 1, 128)
        clean = c.run(kd)
        for s, length in enumerate(c.lengths):
            pos = length - 1
            scales = c.cache.k_scales if spoiled == "k" else c.cache.v_scales
            scales[c.seqs.table[s, pos // 16].long(), :, pos % 16, :, :] = math.nan
        out, lse = c.run(kd)
        last = [4, 6]
        others = [0, 1, 2, 3, 5]
        assert torch.equal(out[others], clean[0][others]) and torch.equal(lse[others], clean[1][others])
        assert out[last].isnan().all()
        assert lse[last].isnan().all() if spoiled == "k" else torch.equal(lse[last], clean[1][last])


def test_bad_pages_are_loud(kd):
    c = Case(kd, [100, 50, 70], [1, 1, 2], 4, 2, 64)
    clean = c.run(kd)
    c.seqs.table[1, 1] = c.cache.pages
    c.seqs.table[2, 4] = -1  # positions 64 ..
    out, lse = c.run(kd)
    assert out[1:].isnan().all() and lse[1:].isnan().all() and torch.equal(out[0], clean[0][0])
    # positions past the table's room
    c.seqs.lengths[0] = c.seqs.table.shape[1] * 16 + 5
    assert c.run(kd)[0][0].isnan().all()
    # a window that does not reach them
    c = Case(kd, [100], [1], 4, 2, 64)
    clean = c.run(kd, window=20)
    c.seqs.table[0, 2] = -5
    assert torch.equal(c.run(kd, window=20)[0], clean[0]) and c.run(kd)[0].isnan().all()


def test_special_queries(kd):
    """An infinity or NaN leaves nothing finite in its row alone."""
    c = Case(kd, [100, 100], [2, 1], 8, 2, 128, dt=BF16)
    clean = c.run(kd)
    c.q[0, 1, 5], c.q[1, 6, 0], c.q[2, 3, 127] = math.nan, math.inf, NONE
    out, lse = c.run(kd)
    bad = torch.zeros(c.q.shape[:2], dtype=torch.bool, device="cuda")
    bad[0, 1] = bad[1, 6] = bad[2, 3] = True
    assert torch.equal(out[~bad], clean[0][~bad]) and torch.equal(lse[~bad], clean[1][~bad])
    assert not torch.isfinite(out[bad]).any()


@pytest.mark.parametrize("size", [2.0 ** -120, 2.0 ** -60, 1e-6, 1e3, 2.0 ** 60, 2.0 ** 125])
def test_queries_of_any_size(kd, size):
    """Powers of two in q that the scale takes off again leave the bits (but in the float's range only)."""
    c = Case(kd, [200], [1], 4, 2, 128, dt=BF16)
    two = 2.0 ** round(math.log2(size))
    plain = c.check(kd, scale=2.0 ** -4)
    c.q = (c.q.double() * two).to(BF16)
    if abs(math.log2(two)) <= 100:
        got = c.run(kd, scale=2.0 ** -4 / two)
        assert torch.allclose(got[0].float(), plain[0].float(), rtol=2.0 ** -7, atol=2.0 ** -8)
    out, lse = c.run(kd, scale=1.0 if two < 1 else 2.0 ** -126)
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()


def test_values_and_scores_that_grow(kd):
    """Steps of values over 24 powers of two and scores that rise along the sequence: every
    rescaling on the way; and the reverse, where none comes after the first."""
    for turn in (False, True):
        c = Case(kd, [1500], [1], 8, 1, 128, page=16, group=64)
        c.lengths = [1500]
        table = c.seqs.table[0].long()
        pos = torch.arange(table.numel() * 16, device="cuda").view(-1, 16)
        if turn:
            pos = pos.flip(0, 1)
        power = (pos // 64 - 12).float()
        c.cache.v_scales[table] = (c.cache.v_scales[table].float() * torch.exp2(power)[:, None, :, None, None]).half()
        c.cache.k_scales[table] = (c.cache.k_scales[table].float() * (0.02 + 0.004 * pos.float())[:, None, :, None, None]).half()
        c.check(kd)
        c.check(kd, scale=0.0)


def test_equal_values(kd):
    """Groups of one value each (step 0), and an all-zero cache."""
    c = Case(kd, [77], [1], 4, 2, 64)
    c.cache.v_scales[..., 0] = 0
    c.check(kd)
    for t in (c.cache.k_scales, c.cache.v_scales):
        t.zero_()
    out, lse = c.run(kd)
    assert (out == 0).all() and torch.allclose(lse, torch.full_like(lse, math.log(77.0)), rtol=1e-6)


def test_layouts(kd):
    """Queries from a projection's rows, unaligned ones, outputs with gaps and head-major: the same bits."""
    c = Case(kd, [90, 40], [2, 3], 6, 2, 64, dt=BF16)
    want = c.check(kd)[0]
    for off, width in ((0, 80), (3, 71)):
        rows = torch.zeros((5, 9, width), dtype=BF16, device="cuda")
        rows[:, :6, off:off + 64] = c.q
        q = rows[:, :6, off:off + 64]
        wide = torch.full((5, 8, 77), 7.0, dtype=BF16, device="cuda")
        kd.attention_4bit(c.cache, q, c.seqs, out=wide[:, 1:7, 5:69])
        assert torch.equal(wide[:, 1:7, 5:69], want)
        wide[:, 1:7, 5:69] = 7
        assert (wide == 7).all()
    major = torch.empty((6, 5, 64), dtype=BF16, device="cuda")
    assert torch.equal(kd.attention_4bit(c.cache, c.q.transpose(0, 1).contiguous().transpose(0, 1), c.seqs, out=major.transpose(0, 1)), want)
    assert torch.equal(kd.attention_4bit(c.cache, c.q, c.seqs), want)
    one = kd.attention_4bit(c.cache, c.q[:, :1].expand(5, 6, 64), c.seqs)
    assert torch.equal(one[:, 0], want[:, 0])


def test_rows_past_most_and_bad_starts(kd):
    c = Case(kd, [60, 40], [4, 2], 4, 2, 64)
    clean, _ = c.run(kd)
    few = kd.Sequences(c.seqs.table, c.seqs.lengths, c.seqs.starts, most=3, longest=60)
    out = torch.full_like(c.q, 7.0)
    kd.attention_4bit(c.cache, c.q, few, out=out)
    assert torch.equal(out[:3], clean[:3]) and (out[3] == 7).all() and torch.equal(out[4:], clean[4:])
    i32 = dict(dtype=torch.int32, device="cuda")
    for starts in ([0, 9, 4], [-2, 1, 3], [0, 4, 2 ** 31 - 1], [2 ** 31 - 1, -2 ** 31, 5], [5, 5, 5]):
        t = kd.Sequences(c.seqs.table, c.seqs.lengths, torch.tensor(starts, **i32), most=3, longest=60)
        out = torch.full_like(c.q, 7.0)
        kd.attention_4bit(c.cache, c.q, t, out=out)
        torch.cuda.synchronize()
    assert (out == 7).all()


def test_workspaces_streams_and_graphs(kd):
    c = Case(kd, [40000, 5000], [1, 1], 8, 2, 128, page=64, dt=BF16)
    want = c.check(kd)
    size = kd.attention_4bit_workspace(c.cache, c.seqs, 8)
    ws = torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda")
    for _ in range(2):  # whatever the workspace holds
        got = c.run(kd, workspace=ws)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    with pytest.raises(kd.KashinError):
        c.run(kd, workspace=ws[:size - 16])
    with pytest.raises(kd.KashinError):
        c.run(kd, workspace=torch.empty(size + 8, dtype=torch.uint8, device="cuda")[8:])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = kd.attention_4bit(c.cache, c.q, c.seqs, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want[0])
    # two captured steps that share a workspace, replayed in turn, lengths moving on
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = kd.attention_4bit(c.cache, c.q, c.seqs, workspace=ws)
        graphs.append((g, out))
    for length in (39999, 64, 1):
        c.seqs.lengths.fill_(length)
        c.q.copy_(torch.randn_like(c.q))
        for g, out in graphs:
            g.replay()
        eager = kd.attention_4bit(c.cache, c.q, c.seqs)
        for _, out in graphs:
            assert torch.equal(out, eager)


def test_a_cache_past_32_bits(kd):
    """Pages whose bytes and words both lie past 2^32."""
    pages = 140000
    cache = kd.new_cache_4bit(pages, 8, 256, 64, 64)
    table = torch.tensor([[pages - 1, 0], [pages // 2, pages - 2]], dtype=torch.int32, device="cuda")
    lengths = torch.tensor([100, 65], dtype=torch.int32, device="cuda")
    x = torch.randn((165, 8, 256), device="cuda").bfloat16()
    starts = torch.tensor([0, 100, 165], dtype=torch.int32, device="cuda")
    kd.cache_write_4bit(cache, x, x.roll(1, 0), kd.Sequences(table, lengths, starts, most=100))
    small = kd.new_cache_4bit(4, 8, 256, 64, 64)
    t = torch.tensor([[1, 3], [0, 2]], dtype=torch.int32, device="cuda")
    kd.cache_write_4bit(small, x, x.roll(1, 0), kd.Sequences(t, lengths, starts, most=100))
    q = torch.randn((2, 16, 256), device="cuda").bfloat16()
    a = kd.attention_4bit(cache, q, kd.Sequences(table, lengths, longest=100))
    b = kd.attention_4bit(small, q, kd.Sequences(t, lengths, longest=100))
    assert torch.equal(a, b) and torch.isfinite(a).all() and a.abs().max() > 0


def test_positions_of_31_bits(kd):
    """The last positions that a sequence may have: what a window sees there is what it sees of the same pages in a
    short sequence (to the bit: the windows start alike in their tiles)."""
    cache = kd.new_cache_4bit(1, 2, 64, 65536, 64)
    x = torch.randn((65536, 2, 64), device="cuda")
    i32 = dict(dtype=torch.int32, device="cuda")
    whole = kd.Sequences(torch.zeros((1, 1), **i32), torch.full((1,), 65536, **i32), most=65536)
    kd.cache_write_4bit(cache, x, x.roll(1, 0), whole)
    q = torch.randn((2, 4, 64), device="cuda").half()
    tables = torch.zeros((1, 2), **i32), torch.zeros((1, 32768), **i32)
    for length, window in ((2 ** 31 - 17, 100), (2 ** 31 - 17, 1), (2 ** 31 - 20, 333), (2 ** 31 - 17, 20000)):
        short = length - (2 ** 31 - 2 * 65536)
        got = []
        for table, n in zip(tables, (short, length)):
            lse = torch.empty((2, 4), dtype=F32, device="cuda")
            s = kd.Sequences(table, torch.full((1,), n, **i32), most=2, longest=window + 1)
            got.append((kd.attention_4bit(cache, q, s, window=window, lse=lse), lse))
        assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
        assert torch.isfinite(got[0][0]).all()
    s = kd.Sequences(tables[1], torch.full((1,), 2 ** 31 - 1, **i32), most=2, longest=100)
    assert kd.attention_4bit(cache, q, s, window=100).isnan().all()


def test_in_place(kd):
    for c in (Case(kd, [300, 2000], [1, 3], 8, 2, 64), Case(kd, [30000, 50], [2, 1], 8, 1, 128, room=200000)):
        want = c.run(kd)[0][:int(c.starts[-1])].clone()
        assert kd.attention_4bit(c.cache, c.q, c.seqs, out=c.q) is c.q
        assert torch.equal(c.q[:int(c.starts[-1])], want)


def test_nothing_to_do(kd):
    cache = kd.new_cache_4bit(2, 2, 64, 16, 64)
    i32 = dict(dtype=torch.int32, device="cuda")
    q = torch.ones((3, 4, 64), dtype=F16, device="cuda")
    out = torch.full_like(q, 5.0)
    kd.attention_4bit(cache, q, kd.Sequences(torch.zeros((0, 1), **i32), torch.zeros(0, **i32)), out=out)
    kd.attention_4bit(cache, q, kd.Sequences(torch.zeros((2, 1), **i32), torch.ones(2, **i32), most=0), out=out)
    assert (out == 5).all()
    assert kd.attention_4bit(cache, q[:0], kd.Sequences(torch.zeros((2, 1), **i32), torch.ones(2, **i32))).shape == (0, 4, 64)
