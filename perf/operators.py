"""Cases of the low-bit serving operators: kd.rmsnorm, kd.matmul_4bit and kd.token_logprobs.

``run`` computes each in its plain form (32-bit torch arithmetic) or, where ``own`` is
true, through the library.  Sizes are those of the library's own 7B-shaped layers (4096,
11008), of a 32,000-token head, and odd ones between.
"""

import math

import torch

own = False

E4M3_MAX = 448.0
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"f16": 2, "bf16": 2, "f32": 4, "e4m3": 1}

# the largest listed cases: what a drawn case may cost at most
MOST_WEIGHTS = 32000 * 4096
MOST_NORM = 2048 * 4096
MOST_LOGITS = 2048 * 32000
MOST_ROWS = 64


def listed():
    norm = {"op": "norm", "residual": True, "y": "none"}
    mat = {"op": "mat4", "group": 128, "zeros": False, "scales": "f16"}
    log = {"op": "logp", "tokens": 1, "masked": False}
    return [
        # one decoded token through the norm before a 7B layer's projections
        dict(norm, name="norm, one token", rows=1, n=4096, x="bf16"),
        # a prompt's rows, with the 16-bit rows that the 2-bit product reads beside the 8-bit ones
        dict(norm, name="norm, a prompt", rows=2048, n=4096, x="bf16", y="bf16"),
        # an odd hidden size without a residual: rows that are not 16-byte aligned
        dict(norm, name="norm, odd rows", rows=333, n=5003, x="f16", residual=False),
        # one decoded token through an attention projection
        dict(mat, name="4-bit q, one token", rows=1, n=4096, m=4096, x="bf16", scales="bf16"),
        # one decoded token through an up projection
        dict(mat, name="4-bit up, one token", rows=1, n=4096, m=11008, x="f16"),
        # sixteen sequences decoded together through a down projection, on the norm's 8-bit rows
        dict(mat, name="4-bit down, 16 rows e4m3", rows=16, n=11008, m=4096, x="e4m3", group=64),
        # an odd layer with zero points, as other quantisers' checkpoints hold them
        dict(mat, name="4-bit odd, zero points", rows=5, n=1367, m=1001, x="f16", group=32, zeros=True),
        # the head for eight sequences decoded together
        dict(mat, name="4-bit head, 8 rows", rows=8, n=4096, m=32000, x="bf16", scales="bf16"),
        # the head for the 64 last positions of a scored window: the largest
        dict(mat, name="4-bit head, 64 rows", rows=64, n=4096, m=32000, x="f16"),
        # one decoded token's log probability with its 20 best alternatives
        dict(log, name="log probabilities, one token", rows=1, vocab=32000, x="f32", top=20),
        # a served batch over an odd vocabulary, tokens masked out, three given tokens each
        dict(log, name="log probabilities, odd and masked", rows=61, vocab=65537, x="f16", top=5, tokens=3, masked=True),
        # perplexity of a 2048-token window: no alternatives wanted but the best one
        dict(log, name="log probabilities, a window", rows=2048, vocab=32000, x="bf16", top=1),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm", "mat4", "mat4", "logp"])
    if op == "norm":
        n = _log_int(rng, 16, 16384)
        n = n // 8 * 8 if rng.random() < 0.6 else n
        return {"op": "norm", "rows": _log_int(rng, 1, min(8192, MOST_NORM // n)), "n": n, "x": rng.choice(["f16", "bf16", "f32"]),
                "residual": rng.random() < 0.7, "y": rng.choice(["none", "f16", "bf16", "f32"])}
    if op == "mat4":
        n = _log_int(rng, 32, 16384)
        n = n // 32 * 32 if rng.random() < 0.6 else n
        return {"op": "mat4", "rows": _log_int(rng, 1, MOST_ROWS), "n": n, "m": _log_int(rng, 16, min(32000, MOST_WEIGHTS // n)),
                "x": rng.choice(["f16", "bf16", "e4m3"]), "group": rng.choice([32, 64, 128]), "zeros": rng.random() < 0.3,
                "scales": rng.choice(["f16", "bf16"])}
    vocab = _log_int(rng, 500, 140000)
    x = rng.choice(["f16", "bf16", "f32"])
    most = MOST_LOGITS * 2 // BYTES[x]
    return {"op": "logp", "rows": _log_int(rng, 1, min(2048, most // vocab)), "vocab": vocab, "x": x, "top": rng.randint(0, 32),
            "tokens": rng.randint(1, 4), "masked": rng.random() < 0.3}


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _activations(g, rows, n):
    """Rows of a model's hidden state: of about unit size, a few channels far larger."""
    a = _randn(g, rows, n)
    big = torch.randint(0, n, (max(1, n // 1000),), generator=g, device="cuda")
    a[:, big] *= 20.0
    return a


def _empty(shape, dtype):
    return torch.empty(shape, dtype=dtype, device="cuda")


def prepare(case, seed):
    g = _gen(seed)
    s = {"case": case}
    if case["op"] == "norm":
        rows, n, dt = case["rows"], case["n"], DTYPES[case["x"]]
        s["x"] = _randn(g, rows, n).to(dt)
        s["weight"] = (1.0 + 0.2 * _randn(g, n)).to(dt)
        s["residual"] = _activations(g, rows, n).to(dt) if case["residual"] else None
        s["new_residual"] = _empty((rows, n), dt) if case["residual"] else None
        s["y"] = None if case["y"] == "none" else _empty((rows, n), DTYPES[case["y"]])
        s["q"] = _empty((rows, n), torch.float8_e4m3fn)
        s["scale"] = _empty((rows,), torch.float32)
    elif case["op"] == "mat4":
        rows, n, m, group = case["rows"], case["n"], case["m"], case["group"]
        groups, nibbles = -(-n // group), -(-n // 32) * 32
        # codes of normally distributed weights, two to a byte, rows of whole 16-byte pieces
        codes = torch.zeros((m, nibbles), dtype=torch.uint8, device="cuda")
        codes[:, :n] = (_randn(g, m, n) * 2.6).round_().add_(8.0).clamp_(0.0, 15.0).to(torch.uint8)
        s["codes"] = (codes[:, 0::2] | (codes[:, 1::2] << 4)).contiguous().view(torch.int32)
        s["scales"] = (torch.exp(0.3 * _randn(g, m, groups)) * 0.008).to(DTYPES[case["scales"]])
        s["zeros"] = torch.randint(5, 11, (m, groups), generator=g, device="cuda").to(torch.uint8) if case["zeros"] else None
        a = _activations(g, rows, n)
        if case["x"] == "e4m3":
            s["x_scale"] = a.abs().amax(1) / E4M3_MAX
            s["x"] = (a / s["x_scale"][:, None]).to(torch.float8_e4m3fn)
        else:
            s["x_scale"], s["x"] = None, a.to(DTYPES[case["x"]])
        s["out"] = _empty((rows, m), torch.float32)
        if own:  # the handle of one layer's weights, which a program keeps
            from paper_2609_11687_gb300 import kashin as kd
            s["w"] = kd.Weight4(s["codes"], s["scales"], s["zeros"], n=n, group=group)
    else:
        rows, vocab, tokens, top = case["rows"], case["vocab"], case["tokens"], case["top"]
        x = _randn(g, rows, vocab) * 3.0
        if case["masked"]:
            x[torch.rand((rows, vocab), generator=g, device="cuda") < 0.2] = -math.inf
            x[1::3, vocab // 2:] = torch.finfo(DTYPES[case["x"]]).min  # the type's lowest value as a mask
            x[2::7] = -math.inf  # rows whose mask leaves nothing
        s["logits"] = x.to(DTYPES[case["x"]])
        s["ids"] = torch.randint(0, vocab, (rows, tokens), generator=g, device="cuda")
        s["ids"][::5, -1] = -1  # no token there
        s["out"] = (_empty((rows, tokens), torch.float32), _empty((rows,), torch.float32), _empty((rows,), torch.float32),
                    _empty((rows, top), torch.int64), _empty((rows, top), torch.float32))
    return s


def _plain_norm(s):
    h = s["x"].float()
    if s["residual"] is not None:
        h = h + s["residual"].float()
    y = h * torch.rsqrt((h * h).mean(1, keepdim=True) + 1e-5) * s["weight"].float()
    a = y.abs().amax(1)
    scale = torch.where(a < 2.0 ** -100, torch.ones_like(a), a / torch.full_like(a, E4M3_MAX))
    out = {"q": (y / scale[:, None]).to(torch.float8_e4m3fn), "scale": scale}
    if s["residual"] is not None:
        out["residual"] = h.to(s["residual"].dtype)
    if s["y"] is not None:
        out["y"] = y.to(s["y"].dtype)
    return out


def _plain_mat4(s):
    n, group = s["case"]["n"], s["case"]["group"]
    b = s["codes"].view(torch.uint8)
    c = torch.stack((b & 15, b >> 4), -1).view(b.shape[0], -1)[:, :n].float()
    c -= 8.0 if s["zeros"] is None else s["zeros"].float().repeat_interleave(group, 1)[:, :n]
    c *= s["scales"].float().repeat_interleave(group, 1)[:, :n]
    y = s["x"].float() @ c.t()
    return y if s["x_scale"] is None else y * s["x_scale"][:, None]


def _plain_logp(s):
    x, ids, top = s["logits"].float(), s["ids"], s["case"]["top"]
    vocab = x.shape[1]
    m = x.amax(1, keepdim=True)
    empty = m == -math.inf
    d = x - torch.where(empty, torch.zeros_like(m), m)
    e = torch.exp(d)
    total = e.sum(1, keepdim=True)
    lse = torch.where(empty, m, m + torch.log(total))
    weighted = torch.where(e > 0, e * d, torch.zeros_like(e)).sum(1, keepdim=True)
    entropy = torch.where(empty, torch.zeros_like(m), torch.log(total) - weighted / total)

    def logp(v):
        return torch.where(empty, torch.full_like(v, -math.inf), v - lse)

    given = logp(x.gather(1, ids.clamp(0, vocab - 1)))
    given = torch.where(ids < 0, torch.zeros_like(given), given)
    # one whole number for each entry: the value's order above, the lowest index below
    bits = (x + 0.0).view(torch.int32)
    key = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long() * 2 ** 32
    key += torch.arange(vocab - 1, -1, -1, device="cuda")
    top_ids = vocab - 1 - (key.topk(top, 1).values & 0xFFFFFFFF) if top else ids.new_empty((x.shape[0], 0))
    return {"logprobs": given, "lse": lse[:, 0], "entropy": entropy[:, 0], "top_ids": top_ids, "top_logprobs": logp(x.gather(1, top_ids))}


def run(state):
    op = state["case"]["op"]
    if not own:
        return {"norm": _plain_norm, "mat4": _plain_mat4, "logp": _plain_logp}[op](state)
    from paper_2609_11687_gb300 import kashin as kd
    if op == "norm":
        r = kd.rmsnorm(state["x"], state["weight"], 1e-5, residual=state["residual"],
                       out=kd.Normed(q=state["q"], scale=state["scale"], y=state["y"], residual=state["new_residual"]))
        out = {"q": r.q, "scale": r.scale, "residual": r.residual, "y": r.y}
        return {k: v for k, v in out.items() if v is not None}
    if op == "mat4":
        return kd.matmul_4bit(state["w"], state["x"], scale=state["x_scale"], out=state["out"])
    r = kd.token_logprobs(state["logits"], state["ids"], state["case"]["top"], out=kd.TokenLogprobs(*state["out"]))
    return {"logprobs": r.logprobs, "lse": r.lse, "entropy": r.entropy, "top_ids": r.top_ids, "top_logprobs": r.top_logprobs}


def work(case):
    if case["op"] == "norm":
        each = 1 + BYTES[case["x"]] * (3 if case["residual"] else 1) + BYTES.get(case["y"], 0)
        return {"bytes": case["rows"] * (case["n"] * each + 4) + case["n"] * BYTES[case["x"]], "flops": 7 * case["rows"] * case["n"]}
    if case["op"] == "mat4":
        rows, n, m = case["rows"], case["n"], case["m"]
        weights = m * (n / 2 + -(-n // case["group"]) * (3 if case["zeros"] else 2))
        return {"bytes": weights + rows * n * BYTES[case["x"]] + 4 * rows * m, "flops": 2 * rows * m * n}
    rows, vocab = case["rows"], case["vocab"]
    return {"bytes": rows * (vocab * BYTES[case["x"]] + case["tokens"] * 12 + case["top"] * 12 + 8), "flops": 6 * rows * vocab}


def exact(case, seed):
    """The definitions in 64 bits."""
    s = prepare(case, seed)
    f64 = torch.float64
    if case["op"] == "norm":
        h = s["x"].to(f64) + (s["residual"].to(f64) if case["residual"] else 0.0)
        root = (h.square().sum(1, keepdim=True) / case["n"] + 1e-5).sqrt()
        y = s["weight"].to(f64) * h / root
        scale = y.abs().max(1).values / E4M3_MAX
        return {"q": y / scale[:, None], "scale": scale, **({"residual": h} if case["residual"] else {}),
                **({} if case["y"] == "none" else {"y": y})}
    if case["op"] == "mat4":
        n, group = case["n"], case["group"]
        x = s["x"].to(f64) * (1.0 if s["x_scale"] is None else s["x_scale"].to(f64)[:, None])
        shifts = torch.arange(0, 32, 4, device="cuda", dtype=torch.int32)
        y = []
        for rows in torch.split(torch.arange(case["m"], device="cuda"), 4000):  # whole at 8 bytes a weight would be large
            c = ((s["codes"][rows][:, :, None] >> shifts) & 15).flatten(1)[:, :n].to(f64)
            which = torch.arange(n, device="cuda") // group
            z = 8.0 if s["zeros"] is None else s["zeros"][rows][:, which].to(f64)
            y.append(torch.einsum("ri,ji->rj", x, s["scales"][rows][:, which].to(f64) * (c - z)))
        return torch.cat(y, 1)
    x = s["logits"].to(f64)
    lse = torch.logsumexp(x, 1, keepdim=True)
    lp = torch.where(lse == -math.inf, lse, x - lse)
    p = lp.exp()
    entropy = -torch.where(p > 0, p * lp, torch.zeros_like(p)).sum(1)
    given = torch.where(s["ids"] < 0, torch.zeros_like(lp[:, :1]), lp.gather(1, s["ids"].clamp(min=0)))
    best = lp.sort(dim=1, descending=True, stable=True).values[:, :case["top"]]
    return {"logprobs": given, "lse": lse[:, 0], "entropy": entropy, "top_ids": None, "top_logprobs": best}
