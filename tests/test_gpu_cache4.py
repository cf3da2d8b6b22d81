"""kd.cache_write_4bit and kd.cache_read_4bit against the quantiser's definition: codes, steps and
lowest values are specified to the bit (IEEE fp32 operations, fp16 rounded outwards), so they are
compared for equality; every value is within half a step of its element."""

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


def _outwards(v, sign):
    """fp16 next to the fp32 values v, towards sign * infinity."""
    with np.errstate(over="ignore"):
        h = v.astype(np.float16)
    inside = h.astype(np.float32) * sign < v * sign
    return np.where(inside, np.nextafter(h, np.float16(sign * np.inf)), h)


def quantise(x, group):
    """Codes, steps and lows (..., groups) of rows x (numpy fp32)."""
    d = x.shape[-1]
    codes, steps, lows = np.zeros(x.shape, dtype=np.int64), [], []
    for a in range(0, d, group):
        part = x[..., a:a + group]
        with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
            low = _outwards(part.min(-1), -1.0)
            step = _outwards((part.max(-1) - low.astype(np.float32)) / np.float32(15), 1.0)
            fine = np.isfinite(low) & np.isfinite(step)
            low, step = (np.where(fine, t, np.float16(np.nan)) for t in (low, step))
            c = np.rint((part - low.astype(np.float32)[..., None]) / step.astype(np.float32)[..., None])
        codes[..., a:a + group] = np.where((fine & (step > 0))[..., None], np.minimum(np.nan_to_num(c), 15), 0)
        steps.append(step)
        lows.append(low)
    return codes, np.stack(steps, -1), np.stack(lows, -1)


def values(codes, steps, lows, group):
    which = np.arange(codes.shape[-1]) // group
    return lows[..., which].astype(np.float32) + steps[..., which].astype(np.float32) * codes.astype(np.float32)


def unpack(words, d):
    w = words.cpu().numpy().view(np.uint32)
    c = np.arange(w.shape[-1] * 8)
    codes = (w[..., c // 8] >> (4 * (c % 8)).astype(np.uint32)) & 15
    assert (codes[..., d:] == 0).all()
    return codes[..., :d].astype(np.int64)


def setup(kd, seqs, longest, most, heads, d, page, group, dt, ragged=True, spare=3, seed=0):
    """A cache of random contents, sequences whose pages lie anywhere, and rows."""
    g = torch.Generator(device="cuda").manual_seed(seed + 31 * d + seqs)
    rng = np.random.RandomState(seed + d + seqs)
    if ragged:
        counts = rng.randint(0, most + 1, seqs)
        lengths = np.maximum(rng.randint(0, longest + 1, seqs), counts)
        counts[0], lengths[0] = most, longest
    else:
        counts, lengths = np.full(seqs, most), np.full(seqs, longest)
    starts = np.concatenate(([0], counts.cumsum()))
    wide = -(-longest // page)
    pages = seqs * wide + 2
    cache = kd.new_cache_4bit(pages, heads, d, page, group)
    for t in (cache.k_codes, cache.v_codes):
        t.copy_(torch.randint(-2 ** 31, 2 ** 31, t.shape, generator=g, device="cuda").int())
    for t in (cache.k_scales, cache.v_scales):
        t.copy_(torch.rand(t.shape, generator=g, device="cuda"))
    table = torch.randperm(pages, generator=g, device="cuda")[:seqs * wide].view(seqs, wide).int()
    s = kd.Sequences(table, torch.from_numpy(lengths).int().cuda(), torch.from_numpy(starts).int().cuda() if ragged else None,
                     most=most, longest=longest)
    tokens = int(starts[-1]) + (spare if ragged else 0)
    rows = (torch.randn((tokens, 2 * heads + 1, d), generator=g, device="cuda") * 2)
    rows[:, :, ::3] += 4
    rows = rows.to(dt)
    return cache, s, rows[:, :heads], rows[:, heads:2 * heads], counts, lengths, starts


def places(table, lengths, counts, starts, page):
    """(row of the call, page, place) of every row that has a place."""
    at = []
    for s, n in enumerate(counts):
        for i in range(n):
            pos = lengths[s] - n + i
            if pos >= 0:
                at.append((starts[s] + i, int(table[s, pos // page]), pos % page))
    return np.array(at).reshape(-1, 3)


@pytest.mark.parametrize("dt", [F16, BF16, F32])
@pytest.mark.parametrize("seqs,longest,most,heads,d,page,group", [
    (1, 1, 1, 1, 128, 16, 64), (4, 100, 30, 3, 80, 16, 32), (3, 70, 5, 8, 128, 64, 128), (40, 33, 2, 2, 64, 32, 64),
    (2, 40, 40, 2, 256, 16, 32), (5, 20, 3, 1, 1, 16, 32), (3, 20, 9, 2, 37, 16, 32), (3, 50, 20, 5, 100, 48, 64),
    (2, 30, 30, 1, 200, 16, 128), (1100, 3, 2, 1, 32, 16, 128), (3, 20, 9, 2, 160, 16, 64)])
def test_write_and_read(kd, seqs, longest, most, heads, d, page, group, dt):
    cache, s, k, v, counts, lengths, starts = setup(kd, seqs, longest, most, heads, d, page, group, dt)
    before = [t.clone() for t in (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales)]
    kd.cache_write_4bit(cache, k, v, s)
    at = places(s.table.cpu().numpy(), lengths, counts, starts, page)
    row, pg, place = at.T
    back = {dtype: kd.cache_read_4bit(cache, s, k.shape[0], dtype, out=tuple(
        torch.full(k.shape, 7.0, dtype=dtype, device="cuda") for _ in range(2))) for dtype in (F16, BF16, F32)}
    for i, (x, words, scales) in enumerate(((k, cache.k_codes, cache.k_scales), (v, cache.v_codes, cache.v_scales))):
        x = x.float().cpu().numpy()[row]
        codes, steps, lows = quantise(x, group)
        assert (unpack(words[pg, :, place], d) == codes).all()
        got = scales[pg, :, place].cpu().numpy()
        assert np.array_equal(got[..., 0], steps) and np.array_equal(got[..., 1], lows)
        val = values(codes, steps, lows, group)
        step = np.repeat(steps.astype(np.float64), group, -1)[..., :d]
        assert (np.abs(val.astype(np.float64) - x) <= step / 2 * (1 + 1e-5) + 1e-6 * np.abs(x)).all()
        # all other places are as they were
        for t, old in ((words, before[2 * i]), (scales, before[2 * i + 1])):
            touched = torch.zeros(t.shape[:3], dtype=torch.bool, device="cuda")
            touched[pg, :, place] = True
            assert torch.equal(t[~touched].view(torch.int16), old[~touched].view(torch.int16))
        for dtype, pair in back.items():
            want = torch.full(k.shape, 7.0, dtype=dtype, device="cuda")
            want[:starts[-1]] = 0.0
            want[torch.from_numpy(row).cuda()] = torch.from_numpy(val).cuda().to(dtype)
            assert torch.equal(pair[i], want), dtype


def test_uniform_rows_and_one_side(kd):
    cache, s, k, v, counts, lengths, starts = setup(kd, 6, 50, 4, 2, 64, 16, 64, F16, ragged=False)
    kd.cache_write_4bit(cache, k, v, s)
    rk, rv = kd.cache_read_4bit(cache, s)
    assert rk.dtype == F16 and rk.shape == k.shape
    only = torch.empty_like(rv)
    assert kd.cache_read_4bit(cache, s, out=(None, only))[0] is None and torch.equal(only, rv)
    assert kd.cache_read_4bit(cache, s, out=(only, None))[1] is None and torch.equal(only, rk)
    # whole sequences as rows of the same cache
    whole = kd.Sequences(s.table, s.lengths, torch.arange(0, 6 * 50 + 1, 50, dtype=torch.int32, device="cuda"), most=50)
    wk, wv = kd.cache_read_4bit(cache, whole, 300)
    assert torch.equal(wk.view(6, 50, 2, 64)[:, 46:].reshape(rk.shape), rk)
    assert torch.equal(wv.view(6, 50, 2, 64)[:, 46:].reshape(rk.shape), rv)


def test_layouts(kd):
    """Head-major rows, odd offsets and gaps: the bits do not go by them."""
    cache, s, k, v, *_ = setup(kd, 3, 40, 7, 4, 64, 16, 32, BF16)
    kd.cache_write_4bit(cache, k, v, s)
    want = [t.clone() for t in (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales)]
    wide = torch.zeros(k.shape[0], 4, 70, dtype=BF16, device="cuda")
    wide[..., 5:69] = k
    kd.cache_write_4bit(cache, wide[..., 5:69], v.transpose(0, 1).contiguous().transpose(0, 1), s)
    for a, b in zip(want, (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales)):
        assert torch.equal(a, b)
    rk, rv = kd.cache_read_4bit(cache, s, k.shape[0], BF16)
    major, gaps = torch.zeros(4, k.shape[0], 64, dtype=BF16, device="cuda").transpose(0, 1), torch.full_like(wide, 3.0)
    kd.cache_read_4bit(cache, s, out=(major, gaps[..., 5:69]))
    n = int(s.starts[-1])
    assert torch.equal(major[:n], rk[:n]) and torch.equal(gaps[:n, :, 5:69], rv[:n])
    assert (gaps[..., :5] == 3).all() and (gaps[..., 69:] == 3).all() and (gaps[n:] == 3).all()
    # a shared key and value head (stride 0)
    one = kd.new_cache_4bit(cache.pages, 4, 64, 16, 32)
    kd.cache_write_4bit(one, k[:, :1].expand_as(k), v[:, :1].expand_as(v), s)
    assert torch.equal(one.k_codes[:, 3], one.k_codes[:, 0])


@pytest.mark.parametrize("dt", [F16, F32])
def test_special_groups(kd, dt):
    """What is no number stays in its group; equal, tiny, large and out of range values."""
    cache = kd.new_cache_4bit(3, 1, 128, 16, 32)
    s = kd.Sequences(torch.tensor([[1]], dtype=torch.int32, device="cuda"), torch.tensor([8], dtype=torch.int32, device="cuda"), most=8)
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((8, 1, 128), generator=g, device="cuda").to(dt)
    x[0, 0, 3], x[1, 0, 40], x[2, 0, 70] = math.nan, math.inf, -math.inf
    x[3, 0, :32], x[3, 0, 32:64], x[3, 0, 64:96] = 0.0, 0.1, -1.5
    x[4] *= 1e-7
    big = 1e30 if dt == F32 else 65504.0
    x[5, 0, :32], x[5, 0, 40], x[5, 0, 70] = 60000.0, big, -big
    x[6, 0, :32] = -0.0
    kd.cache_write_4bit(cache, x, x, s)
    codes, steps, lows = quantise(x.float().cpu().numpy(), 32)
    got = cache.k_scales[1, 0, :8].cpu().numpy()
    assert np.array_equal(got[..., 0], steps[:, 0], equal_nan=True) and np.array_equal(got[..., 1], lows[:, 0], equal_nan=True)
    back = kd.cache_read_4bit(cache, s, dtype=F32)[0].cpu().numpy()
    want = values(codes, steps, lows, 32)
    assert np.array_equal(back, want, equal_nan=True)
    bad = np.zeros((8, 4), dtype=bool)
    bad[0, 0] = bad[1, 1] = bad[2, 2] = True
    if dt == F32:
        bad[5, 1] = bad[5, 2] = True
    assert np.array_equal(np.isnan(back[:, 0]).all(-1), bad.all(-1)) and np.array_equal(np.isnan(back.reshape(8, 4, 32)).all(-1), bad)
    assert np.array_equal(np.isnan(back.reshape(8, 4, 32)).any(-1), bad)


def test_rows_without_a_place(kd):
    """Positions below 0, bad pages, lengths past the table, starts that do not fit: nothing else is touched."""
    cache = kd.new_cache_4bit(4, 2, 64, 16, 64)
    i32 = dict(dtype=torch.int32, device="cuda")
    table = torch.tensor([[0, 1], [2, -1], [3, 9], [-7, 4], [2 ** 31 - 1, 0]], **i32)
    lengths = torch.tensor([1, 18, 35, 3, -5], **i32)
    s = kd.Sequences(table, lengths, most=3)
    x = torch.randn((15, 2, 64), device="cuda").half() + 3
    kd.cache_write_4bit(cache, x, x, s)
    k, v = kd.cache_read_4bit(cache, s)
    assert torch.equal(k.nan_to_num(9.0), v.nan_to_num(9.0))
    kind = [0 if (t == 0).all() else 1 if t.isnan().all() else 2 for t in k]
    #       sequence 0: positions -1, -2 | 1: 15, bad, bad | 2: past the table | 3: bad page | 4: none
    assert kind == [0, 0, 2, 2, 1, 1, 1, 1, 1, 1, 1, 1, 0, 0, 0]
    held = cache.k_scales[..., 0].abs().sum((1, 3)) > 0
    want = torch.zeros_like(held)
    want[0, 0] = want[2, 15] = True
    assert torch.equal(held, want)
    # starts that decrease, or lie past the rows; rows past `most`; a first start above 0
    for starts, rows in (([0, 6, 2, 4, 4, 4], None), ([0, 2, 2, 2, 40, 50], None), ([-3, 1, 2, 2, 2, 2], None), ([2, 3, 3, 3, 3, 3], {2})):
        out = [torch.full_like(x, 5.0) for _ in range(2)]
        t = kd.Sequences(table, lengths, torch.tensor(starts, **i32), most=1)
        kd.cache_read_4bit(cache, t, out=out)
        torch.cuda.synchronize()
        touched = {i for i in range(15) if not (out[0][i] == 5).all()}
        assert touched == rows if rows is not None else len(touched) <= 6


def test_a_cache_past_32_bits(kd):
    """Places whose bytes and words both lie past 2^32."""
    pages = 140000
    cache = kd.new_cache_4bit(pages, 8, 256, 64, 64)
    assert cache.k_codes.numel() > 2 ** 31
    table = torch.tensor([[pages - 1], [0], [pages // 2 + 1]], dtype=torch.int32, device="cuda")
    s = kd.Sequences(table, torch.tensor([64, 5, 20], dtype=torch.int32, device="cuda"), most=5)
    x = torch.randn((15, 8, 256), device="cuda").bfloat16()
    kd.cache_write_4bit(cache, x, -x, s)
    k, v = kd.cache_read_4bit(cache, s, dtype=F32)
    codes, steps, lows = quantise(x.float().cpu().numpy(), 64)
    assert np.array_equal(k.cpu().numpy(), values(codes, steps, lows, 64))
    assert np.array_equal(cache.k_scales[pages - 1, :, 59:64, :, 0].cpu().numpy(), steps[:5].swapaxes(0, 1))
    codes, steps, lows = quantise(-x.float().cpu().numpy(), 64)
    assert np.array_equal(v.cpu().numpy(), values(codes, steps, lows, 64))


def test_nothing_to_do(kd):
    cache = kd.new_cache_4bit(2, 2, 64, 16, 64)
    i32 = dict(dtype=torch.int32, device="cuda")
    none = kd.Sequences(torch.zeros((0, 1), **i32), torch.zeros(0, **i32))
    x = torch.ones((3, 2, 64), dtype=F16, device="cuda")
    kd.cache_write_4bit(cache, x, x, none)
    some = kd.Sequences(torch.zeros((2, 1), **i32), torch.full((2,), 4, **i32), most=0)
    kd.cache_write_4bit(cache, x, x, some)
    kd.cache_write_4bit(cache, x[:0], x[:0], kd.Sequences(torch.zeros((2, 1), **i32), torch.full((2,), 4, **i32)))
    assert not cache.k_codes.any() and not cache.v_scales.any()
    out = torch.full_like(x, 5.0)
    kd.cache_read_4bit(cache, none, out=(out, None))
    assert (out == 5).all()


def test_steps_in_a_graph(kd):
    """A captured step whose lengths move on writes one place after the other, as eager calls do."""
    cache, s, k, v, *_ = setup(kd, 5, 60, 1, 2, 128, 16, 64, BF16, ragged=False)
    other = kd.new_cache_4bit(cache.pages, 2, 128, 16, 64)
    for a, b in ((cache.k_codes, other.k_codes), (cache.k_scales, other.k_scales), (cache.v_codes, other.v_codes), (cache.v_scales, other.v_scales)):
        a.copy_(b)
    kd.cache_write_4bit(cache, k, v, s)
    for a in (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales):
        a.zero_()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kd.cache_write_4bit(cache, k, v, s)
        rk, rv = kd.cache_read_4bit(cache, s, dtype=F32)
    s.lengths.fill_(14)
    for step in range(4):
        s.lengths.add_(1)
        k.copy_(torch.randn_like(k))
        v.copy_(torch.randn_like(v))
        graph.replay()
        kd.cache_write_4bit(other, k, v, s)
        ok, ov = kd.cache_read_4bit(other, s, dtype=F32)
        assert torch.equal(rk, ok) and torch.equal(rv, ov)
    assert torch.equal(cache.k_codes, other.k_codes) and torch.equal(cache.v_scales, other.v_scales)


def test_side_stream(kd):
    cache, s, k, v, *_ = setup(kd, 4, 90, 20, 2, 64, 16, 32, F16)
    kd.cache_write_4bit(cache, k, v, s)
    want = kd.cache_read_4bit(cache, s, k.shape[0])
    n = int(s.starts[-1])
    cache.k_codes.zero_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    kd.cache_write_4bit(cache, k, v, s, stream=side)
    got = kd.cache_read_4bit(cache, s, k.shape[0], stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got[0][:n], want[0][:n]) and torch.equal(got[1][:n], want[1][:n])
