"""Checks of the attention step's operators that need no GPU: the C entry points refuse bad
arguments before any CUDA call, the wrappers bad tensors; rotary tables."""

import ctypes
import math

import numpy as np
import pytest
import torch


@pytest.fixture(scope="module")
def kd():
    from paper_2609_11687_gb300 import build
    build.build()
    from paper_2609_11687_gb300 import kashin
    return kashin


A, NULL = 4096, None  # an aligned address that is never read


def _heads(kd, **k):
    a = dict(x=A, y=A, weight=NULL, heads=2, x_token=128, x_head=64, y_token=128, y_head=64, weight_dtype=kd.KD_F16)
    a.update(k)
    return kd.KdHeads(*a.values())


def _rope(kd, q={}, k=None, **more):
    a = dict(dtype=kd.KD_F16, tokens=3, d=64, positions=A, turns=A, rot=64, layout=0, amplitude=1.0, eps=1e-6)
    a.update(more)
    sides = [_heads(kd, **q), None if k is None else _heads(kd, **k)]
    return kd.kd_rope(*[None if s is None else ctypes.addressof(s) for s in sides], *a.values(), None)


@pytest.mark.parametrize("bad", [
    dict(dtype=3), dict(dtype=9), dict(tokens=-1), dict(tokens=2 ** 31), dict(positions=NULL), dict(turns=NULL),
    dict(positions=A + 4), dict(turns=A + 4), dict(rot=63), dict(rot=0), dict(rot=66), dict(rot=-2), dict(layout=2),
    dict(amplitude=math.inf), dict(amplitude=math.nan), dict(eps=-1.0), dict(eps=math.nan),
    dict(q=dict(x=NULL)), dict(q=dict(y=NULL)), dict(q=dict(x=A + 1)), dict(q=dict(y=A + 1)), dict(q=dict(heads=-1)),
    dict(q=dict(x_token=-1)), dict(q=dict(x_head=-64)), dict(q=dict(y_token=-1)), dict(q=dict(y_head=-1)),
    dict(q=dict(y_head=63)), dict(q=dict(y_token=127)), dict(q=dict(weight=A, weight_dtype=2)), dict(q=dict(weight=A + 1)),
    dict(q=dict(weight=A + 2, weight_dtype=0)), dict(q=dict(heads=2 ** 31)), dict(q=dict(heads=65536)), dict(k=dict(heads=65536), tokens=1), dict(q=dict(heads=2 ** 30, y_token=2 ** 36)),
    dict(k=dict(y_head=63)), dict(k=dict(x=NULL)), dict(k=dict(weight=A, weight_dtype=7))])
def test_rope_refusals(kd, bad):
    assert _rope(kd, **bad) == kd.KD_ERR_INVALID_ARG


def test_rope_lengths_and_nothing_to_do(kd):
    assert _rope(kd, d=0) == kd.KD_ERR_UNSUPPORTED_N
    assert _rope(kd, d=1025) == kd.KD_ERR_UNSUPPORTED_N
    assert _rope(kd, tokens=0, positions=NULL, turns=NULL, q=dict(x=NULL, y=NULL)) == kd.KD_OK
    assert _rope(kd, positions=NULL, turns=NULL, q=dict(x=NULL, y=NULL, heads=0)) == kd.KD_OK
    assert kd.kd_rope(None, None, 1, 3, 64, A, A, 64, 0, 1.0, 1e-6, None) == kd.KD_ERR_INVALID_ARG


def test_rope_turns(kd):
    """The fraction of a turn to within 2^-52 of the whole quotient, and whole turns dropped."""
    f = np.array([1.0, -1.0, 1e-9, -3e-300, 0.0, 12345.678, 2.0 ** 80, math.pi, 1e-25])
    got = np.empty(len(f), dtype=np.uint64)
    assert kd.kd_rope_turns(f.ctypes.data, len(f), got.ctypes.data) == kd.KD_OK
    from fractions import Fraction
    # 2 pi to 60 digits
    two_pi = Fraction(6283185307179586476925286766559005768394338798750211641949889, 10 ** 60)
    for x, t in zip(f, got):
        want = Fraction(float(x)) / two_pi
        off = (Fraction(int(t), 2 ** 64) - want) % 1
        off = min(off, 1 - off)
        assert off <= abs(want) * Fraction(1, 2 ** 52) + Fraction(1, 2 ** 65)
    assert kd.kd_rope_turns(NULL, 1, got.ctypes.data) == kd.KD_ERR_INVALID_ARG
    assert kd.kd_rope_turns(NULL, 0, NULL) == kd.KD_OK
    assert kd.kd_rope_turns(f.ctypes.data, -1, got.ctypes.data) == kd.KD_ERR_INVALID_ARG
    f[3] = math.nan
    assert kd.kd_rope_turns(f.ctypes.data, len(f), got.ctypes.data) == kd.KD_ERR_INVALID_ARG


def test_frequencies(kd):
    f = kd.rotary_frequencies(8, 100.0)
    assert np.allclose(f, [1.0, 100 ** -0.25, 0.1, 100 ** -0.75], rtol=1e-15)
    assert np.allclose(kd.rotary_frequencies(8, 100.0, kd.Scaling("linear", 4.0)), f / 4, rtol=1e-15)
    # bands: pairs of at most 1 and at least 4 turns within 40 positions, one between
    got = kd.rotary_frequencies(8, 100.0, kd.Scaling("bands", 4.0, original=40))
    turns = 40 * f / (2 * math.pi)
    assert turns[0] > 4 and 1 < turns[1] < 4 and turns[2] < 1
    w = (turns[1] - 1) / 3
    assert np.allclose(got, [f[0], f[1] * (w + (1 - w) / 4), f[2] / 4, f[3] / 4], rtol=1e-14)
    # ramp: by index, between the pairs that turn 32 times and once
    s = kd.Scaling("ramp", 4.0, original=4096)
    got, f = kd.rotary_frequencies(128, 10000.0, s), kd.rotary_frequencies(128)
    lo = math.floor(128 * math.log(4096 / (32 * 2 * math.pi)) / (2 * math.log(10000)))
    hi = math.ceil(128 * math.log(4096 / (2 * math.pi)) / (2 * math.log(10000)))
    assert np.allclose(got[:lo + 1], f[:lo + 1]) and np.allclose(got[hi:], f[hi:] / 4) and (np.diff(f / got) >= -1e-12).all()
    assert s.amplitude == pytest.approx(0.1 * math.log(4) + 1) and kd.Scaling("bands", 4.0).amplitude == 1.0


def test_rotation_refusals(kd):
    for bad in (dict(rot=63), dict(rot=0), dict(rot=64, layout="other"), dict(rot=64, base=1.0), dict(rot=64, base=math.inf),
                dict(rot=64, frequencies=np.ones(31)), dict(rot=64, frequencies=np.ones(32), scaling=kd.Scaling("linear", 2.0))):
        with pytest.raises(ValueError):
            kd.Rotation(**bad, device="cpu")
    with pytest.raises(kd.KashinError):
        kd.Rotation(4, frequencies=[1.0, math.nan], device="cpu")
    for bad in (dict(kind="other", factor=2.0), dict(kind="linear", factor=0.0), dict(kind="bands", factor=2.0, low=4.0),
                dict(kind="ramp", factor=math.nan), dict(kind="ramp", factor=2.0, original=0)):
        with pytest.raises(ValueError):
            kd.Scaling(**bad)


def test_rope_wrapper_refuses_host_tensors_and_shapes(kd):
    r = kd.Rotation(64, device="cpu")
    q, at = torch.zeros(3, 2, 64), torch.arange(3)
    with pytest.raises(ValueError, match="CUDA"):
        kd.rope(q, None, at, r)
    with pytest.raises(ValueError, match="positions"):
        kd.rope(q, None, at[:2], r)
    with pytest.raises(ValueError, match="positions"):
        kd.rope(q, None, at.int(), r)
    with pytest.raises(ValueError, match="dtype"):
        kd.rope(q.double(), None, at, r)
    with pytest.raises(ValueError, match="tokens, heads"):
        kd.rope(q[:, 0], None, at, r)


def _cache(kd, **k):
    a = dict(k_codes=A, k_scales=A, v_codes=A, v_scales=A, pages=4, heads=2, page=16, d=64, group=32)
    a.update(k)
    return kd.KdCache4(*a.values())


def _sequences(kd, **k):
    a = dict(table=A, lengths=A, starts=NULL, ld_table=3, seqs=2, wide=3, most=1, longest=48)
    a.update(k)
    return kd.KdSequences(*a.values())


BAD_CACHE = [dict(k_codes=NULL), dict(k_scales=NULL), dict(v_codes=NULL), dict(v_scales=NULL), dict(k_codes=A + 8), dict(k_scales=A + 4),
             dict(v_codes=A + 4), dict(v_scales=A + 2), dict(pages=-1), dict(pages=0), dict(pages=2 ** 31), dict(heads=0), dict(heads=65536),
             dict(page=8), dict(page=24), dict(page=0), dict(page=65552), dict(group=16), dict(group=256)]
BAD_SEQUENCES = [dict(table=NULL), dict(lengths=NULL), dict(table=A + 2), dict(lengths=A + 1), dict(starts=A + 2), dict(ld_table=2),
                 dict(seqs=-1), dict(seqs=2 ** 31), dict(seqs=2 ** 30 + 1), dict(wide=-1), dict(wide=0), dict(wide=2 ** 31, ld_table=2 ** 32), dict(most=-1),
                 dict(most=2 ** 31), dict(longest=-1)]


def _write(kd, cache={}, seqs={}, call="kd_cache_write_4bit", **more):
    a = dict(tokens=2, k=A, k_token=128, k_head=64, v=A, v_token=128, v_head=64, dtype=kd.KD_F16)
    a.update(more)
    c, s = _cache(kd, **cache), _sequences(kd, **seqs)
    return getattr(kd, call)(ctypes.addressof(c), ctypes.addressof(s), *a.values(), None)


@pytest.mark.parametrize("call", ["kd_cache_write_4bit", "kd_cache_read_4bit"])
@pytest.mark.parametrize("bad", [dict(cache=b) for b in BAD_CACHE] + [dict(seqs=b) for b in BAD_SEQUENCES] + [
    dict(tokens=-1), dict(tokens=2 ** 31), dict(tokens=2 ** 30), dict(dtype=3), dict(dtype=-1), dict(k=A + 1), dict(v=A + 1),
    dict(k_token=-1), dict(k_head=-1), dict(v_token=-128), dict(v_head=-64), dict(k=NULL, v=NULL)])
def test_cache_refusals(kd, call, bad):
    assert _write(kd, call=call, **bad) == kd.KD_ERR_INVALID_ARG


def test_cache_calls(kd):
    bad = kd.KD_ERR_INVALID_ARG
    for d in (0, -1, 257):
        assert _write(kd, cache=dict(d=d)) == kd.KD_ERR_UNSUPPORTED_N
        assert _write(kd, cache=dict(d=d), call="kd_cache_read_4bit") == kd.KD_ERR_UNSUPPORTED_N
    assert _write(kd, k=NULL) == bad and _write(kd, v=NULL) == bad
    for over in (dict(k_head=63), dict(k_token=127), dict(v_head=63), dict(v_token=127, v_head=64), dict(v_head=0), dict(k_token=0)):
        assert _write(kd, call="kd_cache_read_4bit", **over) == bad, over
    # nothing to do: no pointer is wanted and no device
    for call in ("kd_cache_write_4bit", "kd_cache_read_4bit"):
        for none in (dict(tokens=0), dict(seqs=dict(seqs=0, table=NULL, lengths=NULL)), dict(seqs=dict(most=0))):
            assert _write(kd, call=call, k=NULL, v=NULL, **none) == kd.KD_OK
        assert getattr(kd, call)(None, None, 0, A, 0, 0, A, 0, 0, 1, None) == bad


def _search(starts, seqs, most, t):
    """The kernels' search for row t's sequence, step by step; every index that it reads is checked."""
    lo, hi = 0, seqs + 1
    while True:
        stride = (hi - lo + 31) // 32
        found = 0
        for lane in range(32):
            at = lo + lane * stride
            if at < hi:
                assert 0 <= at <= seqs
                found += starts[at] <= t
        if found == 0:
            return -1
        lo += (found - 1) * stride
        assert 0 <= lo <= seqs
        if stride == 1:
            break
        hi = min(lo + stride, hi)
        assert hi > lo
    if lo >= seqs:
        return -1
    first, end = starts[lo], starts[lo + 1]
    return -1 if t < first or t >= end or t - first >= most else lo


def test_search_for_a_sequence():
    """Right for starts that do not decrease; in range, and never a row that is not the sequence's, for any."""
    rng = np.random.RandomState(0)
    for seqs in (1, 2, 31, 32, 33, 64, 1000, 1025, 5000):
        counts = rng.randint(0, 4, seqs)
        starts = np.concatenate(([0], counts.cumsum())) + rng.randint(0, 3)
        owner = np.full(starts[-1] + 5, -1)
        for s in range(seqs):
            owner[starts[s]:starts[s + 1]] = s
        for t in rng.randint(0, len(owner), 200):
            assert _search(starts, seqs, 4, t) == owner[t]
        for _ in range(50):
            wild = rng.randint(-5, 50, seqs + 1)
            for t in rng.randint(0, 60, 10):
                s = _search(wild, seqs, 4, t)
                assert s == -1 or wild[s] <= t < min(wild[s + 1], wild[s] + 4)


def test_cache_handles_refuse(kd):
    z, f = torch.zeros((2, 1, 16, 8), dtype=torch.int32), torch.zeros((2, 1, 16, 1, 2)).half()
    with pytest.raises(ValueError, match="group"):
        kd.Cache4(z, f, z, f, d=64, group=48)
    with pytest.raises(ValueError, match="d must"):
        kd.Cache4(z, f, z, f, d=257)
    with pytest.raises(ValueError, match="codes"):
        kd.Cache4(z, f, z, f, d=65)
    with pytest.raises(ValueError, match="page"):
        kd.Cache4(z[:, :, :8], f, z, f, d=64)
    with pytest.raises(ValueError, match="v_codes"):
        kd.Cache4(z, f, z.long(), f, d=64)
    with pytest.raises(ValueError, match="k_scales"):
        kd.Cache4(z, f[..., :1], z, f, d=64)
    with pytest.raises(ValueError, match="CUDA"):
        kd.Cache4(z, f, z, f, d=64)
    t, n = torch.zeros((2, 3), dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    for bad in ((t[0], n), (t, n[:1]), (t, n.long()), (t.t().contiguous().t(), n), (t, n, n), (t, n, torch.zeros(3)), (t, n)):
        with pytest.raises(ValueError):
            kd.Sequences(*bad)


def _attend(kd, cache={}, seqs={}, **more):
    a = dict(tokens=2, heads=4, q=A, q_token=256, q_head=64, dtype=kd.KD_F16, out=A, out_token=256, out_head=64, lse=A, scale=0.125,
             causal=1, window=0, workspace=A, ws_bytes=2 ** 40)
    a.update(more)
    c, s = _cache(kd, **cache), _sequences(kd, **seqs)
    return kd.kd_attention_4bit(ctypes.addressof(c), ctypes.addressof(s), *a.values(), None)


@pytest.mark.parametrize("bad", [dict(cache=b) for b in BAD_CACHE] + [dict(seqs=b) for b in BAD_SEQUENCES] + [
    dict(tokens=-1), dict(tokens=2 ** 31), dict(heads=0), dict(heads=3), dict(heads=-2), dict(heads=2 ** 31), dict(dtype=0), dict(dtype=3),
    dict(q=NULL), dict(out=NULL), dict(q=A + 1), dict(out=A + 1), dict(lse=A + 2), dict(q_token=-1), dict(q_head=-1), dict(out_token=-1),
    dict(out_head=63), dict(out_token=255), dict(out_head=0), dict(scale=math.inf), dict(scale=2.5e38), dict(scale=-2.5e38), dict(scale=math.nan), dict(window=-1),
    dict(window=5, causal=0), dict(window=2 ** 31), dict(seqs=dict(most=2 ** 31 - 1)), dict(seqs=dict(seqs=2 ** 30, most=64))])
def test_attention_refusals(kd, bad):
    assert _attend(kd, **bad) == kd.KD_ERR_INVALID_ARG


def test_attention_calls(kd):
    for d in (0, 257):
        assert _attend(kd, cache=dict(d=d)) == kd.KD_ERR_UNSUPPORTED_N
    long = dict(longest=10 ** 6, wide=10 ** 6, ld_table=10 ** 6)
    c, s = _cache(kd), _sequences(kd, **long)
    size = kd.kd_attention_4bit_workspace(ctypes.addressof(c), ctypes.addressof(s), 4, 0)
    assert size > 0 and size % 16 == 0
    assert _attend(kd, seqs=long, workspace=NULL) == kd.KD_ERR_WORKSPACE
    assert _attend(kd, seqs=long, ws_bytes=size - 1) == kd.KD_ERR_WORKSPACE
    assert _attend(kd, seqs=long, workspace=A + 8) == kd.KD_ERR_WORKSPACE
    assert kd.kd_attention_4bit_workspace(ctypes.addressof(c), ctypes.addressof(s), 3, 0) == 0
    assert kd.kd_attention_4bit_workspace(None, None, 4, 0) == 0
    none = dict(q=NULL, out=NULL, lse=NULL, workspace=NULL)
    assert _attend(kd, tokens=0, **none) == kd.KD_OK
    assert _attend(kd, seqs=dict(seqs=0, table=NULL, lengths=NULL), **none) == kd.KD_OK
    assert _attend(kd, seqs=dict(most=0), **none) == kd.KD_OK
