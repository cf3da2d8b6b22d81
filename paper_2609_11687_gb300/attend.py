"""A decoder's attention step on low-bit weights and a 4-bit cache.

``AttentionStep`` runs the serving operators together as a decoder uses them: ``rmsnorm`` adds the
last block's output to the residual stream and leaves 8-bit rows, ``matmul_4bit`` multiplies them by
the query, key and value projections in one, ``rope`` norms and turns the heads in place,
``cache_write_4bit`` quantises keys and values into the cache, ``attention_4bit`` attends to it and
``matmul_4bit`` projects back.  A prompt, a decoded token and several drafted ones are the same call; the
sequences say which.

    python -m paper_2609_11687_gb300.attend [--prompt P] [--steps S] [--heads H] [--kv-heads K] [--head-size D]

takes a prompt and some decoded tokens through such a step for each size of the cache's groups and prints
how far its attention is from that over the same keys and values in 64 bits, unquantised.
"""

from __future__ import annotations

import argparse

from . import kashin as kd


class AttentionStep:
    """``norm``: the input norm's weight (hidden,); ``qkv``: a Weight4, or the dense matrix to quantise, of the
    query, key and value projections ((heads + 2 kv_heads) d, hidden); ``out``: likewise (hidden, heads d);
    ``cache``: the Cache4 of its keys and values (whose heads and d it goes by); ``rotation``; ``q_norm``,
    ``k_norm``: the head norms' weights (d,), if the model has them; ``eps``: of all its norms."""

    def __init__(self, norm, qkv, out, cache: kd.Cache4, rotation: kd.Rotation, q_norm=None, k_norm=None,
                 eps: float = 1e-5, group: int = 128):
        self.norm, self.cache, self.rotation, self.q_norm, self.k_norm, self.eps = norm, cache, rotation, q_norm, k_norm, eps
        self.qkv = qkv if isinstance(qkv, kd.Weight4) else kd.quantise_4bit(qkv, group)
        self.out = out if isinstance(out, kd.Weight4) else kd.quantise_4bit(out, group)
        d, kv_heads = cache.d, cache.heads
        if norm.shape != (self.qkv.n,) or self.out.m != self.qkv.n:
            raise ValueError(f"the norm's weight and the output projection must have the {self.qkv.n} hidden channels")
        if self.qkv.m % d or self.out.n % d or self.out.n // d % kv_heads or self.qkv.m != self.out.n + 2 * kv_heads * d:
            raise ValueError(f"the projections must be of a multiple of the cache's {kv_heads} heads of {d} channels, and of its keys and values")
        self.heads = self.out.n // d

    def heads_of(self, rows, positions, residual=None, stream=None):
        """Queries, keys and values (tokens, heads, d) of the hidden rows, normed and turned, and the
        rows plus ``residual`` (None without it)."""
        r = kd.rmsnorm(rows, self.norm, self.eps, residual=residual, stream=stream)
        d, h, k = self.cache.d, self.heads, self.cache.heads
        x = kd.matmul_4bit(self.qkv, r.q, scale=r.scale, out_dtype=rows.dtype, stream=stream).view(rows.shape[0], h + 2 * k, d)
        q, key, value = x[:, :h], x[:, h:h + k], x[:, h + k:]
        kd.rope(q, key, positions, self.rotation, self.q_norm, self.k_norm, self.eps, out=(q, key), stream=stream)
        return q, key, value, r.residual

    def step(self, rows, positions, seqs: kd.Sequences, residual=None, window: int = 0, stream=None):
        """The block's output rows (fp32) for the hidden ``rows`` (fp16 or bf16) of the sequences' last
        tokens at ``positions`` (int64), and the new residual.  Writes their keys and values first.  Rows of no sequence, as
        a padded batch has behind the last one, touch nothing of the others', and mean nothing in the output."""
        q, key, value, residual = self.heads_of(rows, positions, residual, stream)
        kd.cache_write_4bit(self.cache, key, value, seqs, stream=stream)
        y = kd.attention_4bit(self.cache, q, seqs, window=window, stream=stream)
        return kd.matmul_4bit(self.out, y.view(y.shape[0], self.out.n), stream=stream), residual


def main(argv=None) -> dict:
    import torch

    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--prompt", type=int, default=500)
    ap.add_argument("--steps", type=int, default=8)
    ap.add_argument("--heads", type=int, default=8)
    ap.add_argument("--kv-heads", type=int, default=2)
    ap.add_argument("--head-size", type=int, default=128)
    ap.add_argument("--seed", type=int, default=0)
    a = ap.parse_args(argv)
    g = torch.Generator(device="cuda").manual_seed(a.seed)
    d, tokens, hidden = a.head_size, a.prompt + a.steps, a.heads * a.head_size

    def randn(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    qkv = (randn((a.heads + 2 * a.kv_heads) * d, hidden) * hidden ** -0.5).half()
    proj = (randn(hidden, hidden) * hidden ** -0.5).half()
    norm, weights = torch.ones(hidden, device="cuda").half(), [(1 + 0.1 * randn(d)).half() for _ in range(2)]
    rows, positions = randn(tokens, hidden).half(), torch.arange(tokens, device="cuda")
    page = 64
    pages = -(-tokens // page)
    table = torch.randperm(pages, generator=g, device="cuda")[None].int()
    lengths = torch.zeros(1, dtype=torch.int32, device="cuda")
    found = {}
    for group in (32, 64, 128):
        step = AttentionStep(norm, qkv, proj, kd.new_cache_4bit(pages, a.kv_heads, d, page, group), kd.Rotation(d),
                             *weights)
        # the prompt in one call, then a token at a time
        parts = [slice(0, a.prompt)] + [slice(i, i + 1) for i in range(a.prompt, tokens)]
        outs = []
        for at in parts:
            q, k, v, _ = step.heads_of(rows[at], positions[at])
            lengths.fill_(at.stop)
            seqs = kd.Sequences(table, lengths, most=at.stop - at.start, longest=tokens)
            kd.cache_write_4bit(step.cache, k, v, seqs)
            outs.append((kd.attention_4bit(step.cache, q, seqs), q, k, v))
        y, q, k, v = (torch.cat(t).double() for t in zip(*outs))
        k, v = (t.repeat_interleave(a.heads // a.kv_heads, 1) for t in (k, v))
        x = torch.einsum("qhd,khd->hqk", q, k) * d ** -0.5
        x = x.masked_fill(positions[None, None] > positions[:, None], -torch.inf)
        want = torch.einsum("hqk,khd->qhd", x.softmax(2), v)
        found[group] = float((y - want).norm() / want.norm())
        print(f"cache in groups of {group:3d}: {4 + 32 / group:.2f} bits a value, attention off by {100 * found[group]:.1f} %")
    return found


if __name__ == "__main__":
    main()
