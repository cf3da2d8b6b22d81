"""A model's last step on low-bit weights: final norm, output head, log probabilities.

``OutputHead`` runs the serving operators together as a decoder uses them: ``rmsnorm`` adds
the last block's output to the residual stream and leaves 8-bit rows with their scales,
``matmul_4bit`` multiplies them by the 4-bit head, ``token_logprobs`` turns the logits into
the log probabilities of the wanted tokens, the entropy and the likeliest alternatives.

    python -m paper_2609_11687_gb300.score [--rows R] [--hidden N] [--vocab V]

scores the same fp16 rows with the dense fp16 head, with the 4-bit head and with that head
decomposed to 2-bit planes (Kashin-DCT; two planes, so four bits a weight as well), and the 4-bit
head on 8-bit rows, and prints the perplexity of each.
"""

from __future__ import annotations

import argparse
import math

from . import kashin as kd


class OutputHead:
    """Final norm and 4-bit output head.  ``head``: a Weight4, or the dense (vocab, hidden)
    matrix to quantise; ``norm``: the norm's weight (hidden,).  ``eight_bits``: the normed rows
    go to the head in e4m3 with a scale each; without it in the hidden rows' own 16-bit type."""

    def __init__(self, norm, head, eps: float = 1e-5, group: int = 128, zeros: bool = False, eight_bits: bool = True):
        self.norm, self.eps, self.eight_bits = norm, eps, eight_bits
        self.head = head if isinstance(head, kd.Weight4) else kd.quantise_4bit(head, group, zeros)
        if norm.shape != (self.head.n,):
            raise ValueError(f"the norm's weight must have the head's {self.head.n} inputs")

    def logits(self, x, residual=None, stream=None):
        """fp32 logits (rows, vocab) of the hidden rows ``x`` (plus ``residual``)."""
        if self.eight_bits:
            r = kd.rmsnorm(x, self.norm, self.eps, residual=residual, stream=stream)
            return kd.matmul_4bit(self.head, r.q, scale=r.scale, stream=stream)
        rows = kd.Normed(y=kd._new(stream, x.shape, x.dtype, x.device))
        r = kd.rmsnorm(x, self.norm, self.eps, residual=residual, out=rows, stream=stream)
        return kd.matmul_4bit(self.head, r.y, stream=stream)

    def score(self, x, ids, residual=None, top: int = 0, stream=None) -> kd.TokenLogprobs:
        """Log probabilities of ``ids`` (int64 (rows,) or (rows, tokens)) after the rows."""
        return kd.token_logprobs(self.logits(x, residual, stream), ids, top, stream=stream)


def perplexity(logprobs) -> float:
    """exp of the mean negative log probability."""
    return math.exp(-logprobs.double().mean().item())


def main(argv=None) -> dict:
    import torch

    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--rows", type=int, default=64)
    ap.add_argument("--hidden", type=int, default=1024)
    ap.add_argument("--vocab", type=int, default=8000)
    ap.add_argument("--seed", type=int, default=0)
    a = ap.parse_args(argv)
    g = torch.Generator(device="cuda").manual_seed(a.seed)

    def randn(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    head = (randn(a.vocab, a.hidden) * a.hidden ** -0.5 * 3).half()
    norm = (1 + 0.1 * randn(a.hidden)).half()
    x, residual = randn(a.rows, a.hidden).half(), randn(a.rows, a.hidden).half()

    # the 16-bit rows that the dense head reads, and tokens drawn from its distribution
    r = kd.rmsnorm(x, norm, residual=residual,
                   out=kd.Normed(y=torch.empty_like(x), residual=torch.empty_like(x)))
    dense = r.y @ head.t()
    ids = torch.multinomial(dense.float().softmax(1), 1, generator=g)
    out = {"dense fp16": perplexity(kd.token_logprobs(dense, ids).logprobs)}

    h4 = OutputHead(norm, head, eight_bits=False)
    out["4 bits"] = perplexity(h4.score(x, ids, residual).logprobs)
    out["4 bits, 8-bit rows"] = perplexity(OutputHead(norm, h4.head).score(x, ids, residual).logprobs)

    d = kd.decompose(head, iters=16, sign_seed=1)
    xp = kd.apply_p(r.y.float(), 1).half()
    out["2-bit planes"] = perplexity(kd.token_logprobs(kd.matmul_2bit_f16(d, r.y, xp), ids).logprobs)
    for name, value in out.items():
        print(f"{name:18s} perplexity {value:.3f}")
    return out


if __name__ == "__main__":
    main()
