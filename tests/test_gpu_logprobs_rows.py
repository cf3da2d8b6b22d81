"""kd.token_logprobs on more rows than a launch has CTAs (2^20), so that some take a second one,
against the formulas in 64 bits.

Tolerances, with u = 2^-24, for at most 64 entries: S adds at most 8 terms in a thread and
joins 13 times with two roundings each; a term has the power's 2^-21: e = 34 u + 2^-21.  lse,
log probabilities: e + 2 u (|lse| + ln S + 1), u of themselves more; entropy: 4 e (1 + H) + 4 u (ln S + 1)."""

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module")
def kd():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2609_11687_gb300 import build
    build.build()
    from paper_2609_11687_gb300 import kashin
    return kashin


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("top", [0, 1, 5])
def test_more_rows_than_ctas(kd, dt, top):
    g = torch.Generator(device="cuda").manual_seed(top)
    rows, vocab = 2 ** 20 + 3001, 21
    x = (torch.randn((rows, vocab), generator=g, device="cuda") * 3).to(dt)
    x[::5, 3] = -torch.inf
    x[::101] = -torch.inf          # nothing left
    x[7::103] = 0.5                # equal values
    x[11::107, 20] = torch.nan
    ids = torch.randint(0, vocab, (rows, 2), generator=g, device="cuda")
    ids[::3, 1] = -1
    r = kd.token_logprobs(x, ids, top)
    x64 = x.double()
    nan = x64.isnan().any(1)
    none = (x64 == -torch.inf).all(1)
    m = x64.amax(1, keepdim=True)
    d = torch.where(none[:, None], x64, x64 - m)
    log_s = d.exp().sum(1, keepdim=True).log()
    lse = torch.where(none, m[:, 0], (m + log_s)[:, 0])
    lp = torch.where(none[:, None], m, d - log_s)
    p = lp.exp()
    entropy = -torch.where(p > 0, p * lp, torch.zeros_like(p)).sum(1)
    e = 34 * U + 2.0 ** -21
    log_s = torch.where(none[:, None], torch.zeros_like(log_s), log_s)[:, 0]
    tol = e + 2 * U * (torch.where(none, torch.zeros_like(lse), lse).abs() + log_s + 1)

    def near(a, b, t):
        a = a.double()
        return ((a == b) | ((a - b).abs() <= t))[~nan].all()

    assert near(r.lse, lse, tol) and near(r.entropy, entropy, 4 * e * (1 + entropy) + 4 * U * (log_s + 1))
    given = lp.gather(1, ids.clamp(min=0))
    given = torch.where(ids < 0, torch.zeros_like(given), given)
    assert near(r.logprobs, given, tol[:, None] + U * given.abs())
    assert r.lse[nan].isnan().all() and r.entropy[nan].isnan().all() and (r.top_ids[nan] == -1).all()
    if top:
        order = x64.sort(dim=1, descending=True, stable=True).indices[:, :top]
        assert torch.equal(r.top_ids[~nan], order[~nan])
        want = lp.gather(1, order)
        assert near(r.top_logprobs, want, tol[:, None] + U * want.abs())
