"""The attention step's whole path (rmsnorm -> matmul_4bit -> rope -> cache_write_4bit -> attention_4bit
-> matmul_4bit) as a program runs it: prompts, decoded and drafted tokens of several sequences against 64
bits from the path's own projections, in a CUDA graph, and the example."""

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


def _step(kd, hidden, heads, kv_heads, d, dt, page=16, group=64, pages=40, rot=None):
    from paper_2609_11687_gb300.attend import AttentionStep
    g = torch.Generator(device="cuda").manual_seed(hidden + d)

    def randn(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    qkv = (randn((heads + 2 * kv_heads) * d, hidden) * hidden ** -0.5).to(dt)
    out = (randn(hidden, heads * d) * (heads * d) ** -0.5).to(dt)
    norms = [(1 + 0.1 * randn(n)).to(dt) for n in (hidden, d, d)]
    step = AttentionStep(norms[0], qkv, out, kd.new_cache_4bit(pages, kv_heads, d, page, group), kd.Rotation(rot or d), *norms[1:])
    return step, randn


def _sequences(kd, lengths, counts, page, table):
    starts = torch.zeros(len(counts) + 1, dtype=torch.int32, device="cuda")
    starts[1:] = torch.tensor(counts, device="cuda").cumsum(0)
    positions = torch.cat([torch.arange(n - c, n) for n, c in zip(lengths, counts)]).cuda()
    return kd.Sequences(table, torch.tensor(lengths, dtype=torch.int32, device="cuda"), starts, most=max(counts), longest=max(lengths)), positions


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("hidden,heads,kv_heads,d,rot", [(256, 4, 2, 64, 64), (384, 3, 3, 128, 32), (320, 8, 1, 80, 80)])
def test_prompt_then_tokens(kd, hidden, heads, kv_heads, d, rot, dt):
    """Against 64 bits from the path's own queries and what its cache holds.  An output of the attention is off
    by half a step of its type and by the rounding of weights, 2^-11 of a value's range, which is at
    most 8 of 15 steps from its middle; what is compared is within twice half a step of the largest value.  The
    projection back adds fp32 sums (2e-5 of the largest row sum is far above them)."""
    step, randn = _step(kd, hidden, heads, kv_heads, d, dt, rot=rot)
    page = step.cache.page
    table = torch.randperm(40, device="cuda")[:36].view(3, 12).int()
    lengths = [0, 0, 0]
    eps = torch.finfo(dt).eps
    for counts in ([50, 7, 0], [1, 1, 1], [3, 1, 5], [1, 0, 90]):
        lengths = [n + c for n, c in zip(lengths, counts)]
        seqs, positions = _sequences(kd, lengths, counts, page, table)
        x, residual = randn(sum(counts), hidden).to(dt), randn(sum(counts), hidden).to(dt)
        y, new = step.step(x, positions, seqs, residual=residual)
        assert torch.equal(new, (x.float() + residual.float()).to(dt))
        q, k, v, _ = step.heads_of(x, positions, residual)
        rk, rv = kd.cache_read_4bit(step.cache, seqs, sum(counts), torch.float32)
        for kept, made in ((rk, k.float()), (rv, v.float())):  # half a step of the cache
            part = made.reshape(*made.shape[:2], -1)
            spread = part.amax(2) - part.amin(2)
            assert ((kept - made).abs() <= (spread / 30 * 1.01 + 1e-3)[..., None]).all()
        at, want = 0, []
        whole = kd.Sequences(table, seqs.lengths, torch.tensor([0, *torch.tensor(lengths).cumsum(0).tolist()], dtype=torch.int32, device="cuda"), most=max(lengths))
        ak, av = (t.double() for t in kd.cache_read_4bit(step.cache, whole, sum(lengths), torch.float32))
        first, top = 0, av.abs().max()
        for n, c in zip(lengths, counts):
            keys, values = (t[first:first + n].repeat_interleave(heads // kv_heads, 1) for t in (ak, av))
            s = torch.einsum("qhd,khd->hqk", q[at:at + c].double(), keys) * d ** -0.5
            own = torch.arange(n - c, n, device="cuda")[:, None]
            s = s.masked_fill(torch.arange(n, device="cuda") > own, -torch.inf)
            want.append(torch.einsum("hqk,khd->qhd", s.softmax(2), values))
            at, first = at + c, first + n
        want = torch.cat(want)
        got = kd.attention_4bit(step.cache, q, seqs)
        assert ((got.double() - want).abs() <= eps / 2 * want.abs() + (2.0 ** -10 + 1e-5) * top).all()
        back = got.double().reshape(len(got), -1) @ kd.dequantise_4bit(step.out).double().t()
        assert (y.double() - back).abs().max() <= 2e-5 * back.abs().max()


def test_drafted_tokens_are_decoded_tokens(kd):
    """Several tokens of a sequence in one call leave, to the products' rounding and a code of the cache, the outputs and
    the cached rows of as many calls of one."""
    step, randn = _step(kd, 256, 4, 2, 64, torch.float16)
    other, _ = _step(kd, 256, 4, 2, 64, torch.float16)
    table = torch.randperm(40, device="cuda")[:24].view(2, 12).int()
    x = randn(2 * 60, 256).half().view(2, 60, 256)
    seqs, positions = _sequences(kd, [50, 50], [50, 50], 16, table)
    for s in (step, other):
        s.step(x[:, :50].reshape(100, 256), positions, seqs)
    seqs, positions = _sequences(kd, [60, 60], [10, 10], 16, table)
    y, _ = step.step(x[:, 50:].reshape(20, 256), positions, seqs)
    for i in range(50, 60):
        seqs, positions = _sequences(kd, [i + 1, i + 1], [1, 1], 16, table)
        one, _ = other.step(x[:, i].contiguous(), positions, seqs)
        # up to 8 rows the products before share their order of sums with 20 rows' only to fp32's last places
        assert (one - y.view(2, 10, 256)[:, i - 50]).abs().max() <= 2e-2 * y.abs().max()
    assert (kd.cache_read_4bit(step.cache, kd.Sequences(table, seqs.lengths, most=60))[0].float()
            - kd.cache_read_4bit(other.cache, kd.Sequences(table, seqs.lengths, most=60))[0].float()).abs().max() <= 0.5


def test_decoding_in_a_graph(kd):
    """One captured step, replayed while its lengths and positions move on, gives the eager bits, and
    leaves the eager cache."""
    step, randn = _step(kd, 256, 8, 2, 64, torch.bfloat16)
    other, _ = _step(kd, 256, 8, 2, 64, torch.bfloat16)
    table = torch.randperm(40, device="cuda")[:36].view(3, 12).int()
    lengths = torch.tensor([31, 1, 100], dtype=torch.int32, device="cuda")
    seqs = kd.Sequences(table, lengths)
    x, positions = randn(3, 256).bfloat16(), (lengths - 1).long()
    step.step(x, positions, seqs)
    torch.cuda.synchronize()
    for t in ("k_codes", "k_scales", "v_codes", "v_scales"):
        getattr(step.cache, t).copy_(getattr(other.cache, t))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, _ = step.step(x, positions, seqs)
    for t in ("k_codes", "k_scales", "v_codes", "v_scales"):
        getattr(step.cache, t).copy_(getattr(other.cache, t))
    for _ in range(20):
        x.copy_(randn(3, 256))
        graph.replay()
        want, _ = other.step(x, positions, seqs)
        assert torch.equal(y, want)
        lengths.add_(1)
        positions.add_(1)
    for t in ("k_codes", "k_scales", "v_codes", "v_scales"):
        assert torch.equal(getattr(step.cache, t), getattr(other.cache, t))


def test_side_stream(kd):
    step, randn = _step(kd, 256, 4, 2, 64, torch.float16)
    table = torch.randperm(40, device="cuda")[:12].view(1, 12).int()
    seqs, positions = _sequences(kd, [40], [40], 16, table)
    x = randn(40, 256).half()
    want, _ = step.step(x, positions, seqs)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got, _ = step.step(x, positions, seqs, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)


def test_refusals(kd):
    from paper_2609_11687_gb300.attend import AttentionStep
    step, randn = _step(kd, 256, 4, 2, 64, torch.float16)
    for norm, qkv, out in ((step.norm[:128], step.qkv, step.out), (step.norm, step.qkv, step.qkv), (step.norm, step.out, step.out)):
        with pytest.raises(ValueError):
            AttentionStep(norm, qkv, out, step.cache, step.rotation)


def test_example(kd):
    from paper_2609_11687_gb300 import attend
    found = attend.main(["--prompt", "100", "--steps", "3", "--heads", "4", "--kv-heads", "2", "--head-size", "64"])
    assert set(found) == {32, 64, 128} and all(0 < v < 1 for v in found.values())
