"""kd.token_logprobs against its formulas in 64 bits; the alternatives' ids exactly.

Tolerances, with u = 2^-24: S = sum e^(x - m) adds at most vocab / 512 terms in a thread and
joins at most 13 times with two roundings each; a term has the power's 2^-21 (2 units, and
the rounding of its argument, which e^d |d| <= 0.37 bounds): S is off by
e = (vocab / 512 + 64) u + 2^-21 relative.  lse = m + ln S: e + 2 u (|lse| + ln S + 1) absolute,
a log probability that and u of itself.  The entropy ln S - T / S, T = sum e^d d with terms of
one sign: 4 e (1 + H) + 4 u (ln S + 1)."""

import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
INF = math.inf
TYPES = [torch.float16, torch.bfloat16, torch.float32]


@pytest.fixture(scope="module")
def kd():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2609_11687_gb300 import build
    build.build()
    from paper_2609_11687_gb300 import kashin
    return kashin


def _near(a, b, tol):
    a = a.double()
    same = (a == b) | (a.isnan() & b.isnan())
    return (same | ((a - b).abs() <= tol)).all()


def _check(logits, ids, top, r):
    x = logits.double()
    vocab = x.shape[1]
    m = x.amax(1, keepdim=True)
    # relative to the maximum: beside 3e38 a logarithm of the vocabulary is lost in 64 bits too
    d = torch.where(m == -INF, x, x - m)
    log_s = d.exp().sum(1, keepdim=True).log()
    lse = torch.where(m == -INF, m, m + log_s)
    lp = torch.where(m == -INF, m, d - log_s)
    p = lp.exp()
    entropy = -torch.where(p > 0, p * lp, torch.zeros_like(p)).sum(1)
    e = (vocab / 512 + 64) * U + 2.0 ** -21
    log_s = torch.where(lse.isfinite(), log_s, torch.zeros_like(m))
    tol = e + 2 * U * (lse.abs() + log_s + 1)
    assert _near(r.lse, lse[:, 0], tol[:, 0])
    assert _near(r.entropy, entropy, 4 * e * (1 + entropy) + 4 * U * (log_s[:, 0] + 1))
    ids = ids.view(x.shape[0], -1)
    given = lp.gather(1, ids.clamp(0, vocab - 1))
    given = torch.where(ids < 0, torch.zeros_like(given), given)
    assert _near(r.logprobs, given, tol + U * given.abs())
    if top:
        # descending, equal values by lowest id (-0 counts as 0)
        order = (x + 0.0).sort(dim=1, descending=True, stable=True).indices[:, :top]
        assert torch.equal(r.top_ids, order)
        want = lp.gather(1, order)
        assert _near(r.top_logprobs, want, tol + U * want.abs())


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("rows,vocab,top", [
    (1, 1, 1), (2, 2, 2), (3, 7, 7), (1, 31, 0), (4, 33, 32), (2, 500, 20), (1, 4096, 1), (5, 4097, 3), (1, 32000, 20), (2, 65537, 32),
    (1, 131072, 32), (310, 9001, 5), (1, 300001, 8)])
def test_against_64_bits(kd, dt, rows, vocab, top):
    g = torch.Generator(device="cuda").manual_seed(vocab + rows)
    logits = (torch.randn((rows, vocab), generator=g, device="cuda") * 3).to(dt)
    ids = torch.randint(0, vocab, (rows, 3), generator=g, device="cuda")
    ids[0, 0] = -1
    r = kd.token_logprobs(logits, ids, top)
    _check(logits, ids, top, r)
    r2 = kd.token_logprobs(logits, ids, top)
    for a, b in zip(vars(r).values(), vars(r2).values()):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("rows,vocab", [(3, 40), (2, 32000), (400, 5001)])
def test_ties(kd, dt, rows, vocab):
    """Rows of equal values, of a few values, and with zeros of both signs: ids by lowest
    index."""
    g = torch.Generator(device="cuda").manual_seed(vocab)
    top = 32
    few = torch.randint(0, 3, (rows, vocab), generator=g, device="cuda").to(dt)
    few[0] = 2.5
    few[-1] = torch.where(torch.rand(vocab, generator=g, device="cuda") < 0.5, 0.0, -0.0).to(dt)
    ids = torch.zeros((rows, 1), dtype=torch.int64, device="cuda")
    _check(few, ids, top, kd.token_logprobs(few, ids, top))


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("rows,vocab", [(5, 100), (5, 32768), (320, 3000)])
def test_masks(kd, dt, rows, vocab):
    """-infinity and the type's lowest value as masks: some entries, all but one, all."""
    g = torch.Generator(device="cuda").manual_seed(vocab + 1)
    x = (torch.randn((rows, vocab), generator=g, device="cuda") * 4).to(dt)
    low = torch.finfo(dt).min
    x[0, torch.rand(vocab, generator=g, device="cuda") < 0.9] = -INF
    x[1, torch.rand(vocab, generator=g, device="cuda") < 0.9] = low
    x[2] = -INF
    x[3] = low
    x[4] = -INF
    x[4, vocab - 1] = 1.5
    ids = torch.randint(0, vocab, (rows, 2), generator=g, device="cuda")
    r = kd.token_logprobs(x, ids, 12)
    _check(x, ids, 12, r)
    assert r.entropy[2] == 0 and r.lse[2] == -INF and r.top_ids[2].tolist() == list(range(12))
    assert abs(r.entropy[3].item() - math.log(vocab)) < 1e-4
    assert r.top_ids[4, 0] == vocab - 1 and r.entropy[4] == 0 and r.top_logprobs[4, 0] == 0


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("vocab", [50, 40000])
def test_nan_and_infinity(kd, dt, vocab):
    x = torch.randn((4, vocab), device="cuda").to(dt)
    clean = x.clone()
    x[1, vocab // 2] = float("nan")
    x[2, 3] = INF
    ids = torch.tensor([[0, vocab, -5]] * 4, device="cuda")
    r = kd.token_logprobs(x, ids, 3)
    assert r.lse[1].isnan() and r.entropy[1].isnan() and r.logprobs[1, 0].isnan() and r.top_logprobs[1].isnan().all()
    assert (r.top_ids[1] == -1).all()
    assert r.lse[2] == INF and r.entropy[2].isnan() and r.logprobs[2, 0].isnan() and r.top_ids[2, 0] == 3
    assert r.logprobs[:, 1].isnan().all() and (r.logprobs[:, 2] == 0).all()  # past the vocabulary; padding
    ref = kd.token_logprobs(clean, ids, 3)
    for k in (0, 3):
        for a, b in zip(vars(r).values(), vars(ref).values()):
            assert torch.equal(a[k].nan_to_num(9.0) if a.is_floating_point() else a[k],
                               b[k].nan_to_num(9.0) if b.is_floating_point() else b[k])


@pytest.mark.parametrize("dt", TYPES)
def test_alternatives_crowded_in_few_pieces(kd, dt):
    """The largest values all lie where the same few threads read: more of them reach the
    bar than fit the list at once."""
    piece = 4 if dt == torch.float32 else 8
    vocab, rows = 32768 * 2, 310
    x = torch.randn((rows, vocab), device="cuda").to(dt)
    owner = (torch.arange(vocab, device="cuda") // piece) % 512
    big = torch.rand(vocab, device="cuda") * 4 + 20
    x[7] = torch.where(owner < 31, big, x[7].float()).to(dt)
    x[9] = torch.where((owner % 256) < 31, big, x[9].float()).to(dt)
    ids = torch.zeros((rows, 1), dtype=torch.int64, device="cuda")
    _check(x, ids, 32, kd.token_logprobs(x, ids, 32))


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("off,pad", [(0, 8), (1, 2), (3, 5), (0, 1)])
def test_strides_and_alignment(kd, dt, off, pad):
    rows, vocab = 6, 5000
    buf = torch.full((off + rows * (vocab + pad),), 99.0, dtype=dt, device="cuda")  # larger than any logit
    x = buf[off:].view(rows, vocab + pad)[:, :vocab]
    x.copy_(torch.randn((rows, vocab), device="cuda"))
    ids = torch.randint(0, vocab, (rows,), device="cuda")
    _check(x, ids, 9, kd.token_logprobs(x, ids, 9))


def test_large_offsets(kd):
    """Rows past 2^32 bytes and 2^31 elements."""
    ld = 2 ** 30 + 3
    buf = torch.empty(2 * ld + 6000, dtype=torch.float16, device="cuda")
    x = buf.as_strided((3, 6000), (ld, 1))
    x.copy_(torch.randn((3, 6000), device="cuda"))
    ids = torch.randint(0, 6000, (3, 1), device="cuda")
    _check(x, ids, 4, kd.token_logprobs(x, ids, 4))


def test_optional_outputs_streams_and_refusals(kd):
    x = torch.randn((3, 1000), device="cuda")
    ids = torch.randint(0, 1000, (3, 2), device="cuda")
    ref = kd.token_logprobs(x, ids, 4)
    out = kd.TokenLogprobs(torch.empty_like(ref.logprobs), None, None, torch.empty_like(ref.top_ids), torch.empty_like(ref.top_logprobs))
    kd.token_logprobs(x, ids, 4, out=out)
    assert torch.equal(out.logprobs, ref.logprobs) and torch.equal(out.top_ids, ref.top_ids)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    a = kd.token_logprobs(x, ids, 4, stream=s)
    with torch.cuda.stream(s):
        b = kd.token_logprobs(x, ids, 4)
    s.synchronize()
    for r in (a, b):
        assert all(torch.equal(u, v) for u, v in zip(vars(r).values(), vars(ref).values()))
    none = kd.token_logprobs(x, ids[:, :0], 0)
    assert none.logprobs.shape == (3, 0) and torch.equal(none.lse, ref.lse) and torch.equal(none.entropy, ref.entropy)
    assert kd.token_logprobs(x[:0], ids[:0], 4).top_ids.shape == (0, 4)
    for bad in (dict(top=33), dict(top=-1)):
        with pytest.raises(ValueError, match="top"):
            kd.token_logprobs(x, ids, **bad)
    with pytest.raises(ValueError, match="ids"):
        kd.token_logprobs(x, ids.int())
    with pytest.raises(ValueError, match="ids"):
        kd.token_logprobs(x, ids[:2])
    with pytest.raises(ValueError, match="out.lse"):
        kd.token_logprobs(x, ids, 0, out=kd.TokenLogprobs(ref.logprobs, ref.lse[:2], None, none.top_ids, none.top_logprobs))


def test_graph_capture(kd):
    """The calls only enqueue work: they can be captured and replayed on new values."""
    x = torch.randn((2, 3000), device="cuda")
    ids = torch.randint(0, 3000, (2, 1), device="cuda")
    out = kd.token_logprobs(x, ids, 5)
    torch.cuda.synchronize()
    gr = torch.cuda.CUDAGraph()
    with torch.cuda.graph(gr):
        kd.token_logprobs(x, ids, 5, out=out)
    x.copy_(torch.randn((2, 3000), device="cuda"))
    gr.replay()
    torch.cuda.synchronize()
    _check(x, ids, 5, out)
