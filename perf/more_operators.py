"""Cases of the attention step's operators on low bits: kd.rope (head norms and rotary positions),
kd.cache_write_4bit / kd.cache_read_4bit (a paged key and value cache of 4-bit codes) and
kd.attention_4bit (attention over that cache).

``run`` computes each in its plain form (32-bit torch arithmetic, angles in 64) or, where
``own`` is true, through the library.  Heads are those of the library's own 7B-shaped layers
(4096 = 32 x 128), with as many or fewer key heads, and odd ones.
"""

import math

import numpy as np
import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"f16": 2, "bf16": 2, "f32": 4}

# the largest listed cases: what a drawn case may cost at most
MOST_ROPE = 2048 * 40 * 128
MOST_STORE = 2000 * 8 * 128
MOST_READ = 8 * 4096 * 8 * 128
MOST_ATTENTION = 32 * 8192 * 8 * 128


def listed():
    rope = {"op": "rope", "base": 10000.0, "scaling": "none", "layout": "half", "norm": False, "far": 4096}
    cache = {"page": 64, "group": 64, "spare": 0, "ragged": False}
    store = dict(cache, op="store", most=1)
    read = dict(cache, op="read")
    att = dict(cache, op="attention", most=1, window=0, causal=True)
    return [
        # one decoded token of a 7B layer with fewer key heads
        dict(rope, name="rope, one token", tokens=1, hq=32, hk=8, d=128, rot=128, x="bf16"),
        # a prompt's rows, with the norm of each head before its rotation
        dict(rope, name="rope, a prompt with norms", tokens=2048, hq=32, hk=8, d=128, rot=128, x="bf16", norm=True),
        # part of an odd head, neighbours paired, far positions of a stretched context
        dict(rope, name="rope, odd heads, far", tokens=333, hq=10, hk=2, d=80, rot=32, x="f16", layout="interleaved",
             scaling="bands", base=500000.0, far=1000000),
        # eight sequences' decoded tokens go to the cache
        dict(store, name="store, 8 tokens", seqs=8, longest=4096, hk=8, d=128, x="f16"),
        # pieces of four prompts of unlike lengths, written together
        dict(store, name="store, pieces of prompts", seqs=4, longest=4096, most=500, hk=8, d=128, x="bf16", ragged=True),
        # whole sequences read back, for a dense product over a long prompt
        dict(read, name="read, whole sequences", seqs=8, longest=4096, hk=8, d=128, x="bf16", ragged=True),
        # odd heads, small groups and pages
        dict(read, name="read, odd heads", seqs=5, longest=777, hk=3, d=80, x="f32", group=32, page=16, ragged=True),
        # one token of one sequence, a 7B layer with all its key heads: the smallest
        dict(att, name="attention, one sequence", seqs=1, longest=1001, hq=32, hk=32, d=128, x="f16"),
        # one token of a long document
        dict(att, name="attention, a long document", seqs=1, longest=131072, hq=32, hk=8, d=128, x="bf16"),
        # a served batch of unlike lengths: the largest
        dict(att, name="attention, 32 sequences", seqs=32, longest=8192, hq=32, hk=8, d=128, x="bf16", ragged=True),
        # odd heads under a sliding window, one sequence still empty
        dict(att, name="attention, odd heads, window", seqs=7, longest=2500, hq=15, hk=3, d=80, x="f16", group=32, page=16,
             window=1000, ragged=True),
        # eight drafted tokens of each sequence checked at once, and rows of padding behind them
        dict(att, name="attention, drafted tokens", seqs=16, longest=4096, most=8, hq=32, hk=8, d=128, x="bf16", group=128,
             ragged=True, spare=5),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rope", "store", "read", "attention", "attention"])
    d = rng.choice([64, 128, 128, 256, rng.randint(8, 128) * 2])
    if op == "rope":
        hk = rng.randint(1, 16)
        hq = hk * rng.choice([1, 2, 4, 7])
        rot = d if rng.random() < 0.6 else rng.randint(1, d // 2) * 2
        return {"op": "rope", "tokens": _log_int(rng, 1, max(1, MOST_ROPE // ((hq + hk) * d))), "hq": hq, "hk": hk, "d": d, "rot": rot,
                "x": rng.choice(["f16", "bf16", "f32"]) if hq * d < 4000 else rng.choice(["f16", "bf16"]),
                "layout": rng.choice(["half", "interleaved"]), "norm": rng.random() < 0.5, "base": rng.choice([10000.0, 500000.0]),
                "scaling": rng.choice(["none", "linear", "bands", "ramp"]), "far": _log_int(rng, 16, 1000000)}
    case = {"op": op, "page": rng.choice([16, 32, 64, 128]), "group": rng.choice([32, 64, 128]), "d": d, "ragged": rng.random() < 0.6,
            "hk": rng.choice([1, 2, 3, 4, 8, 16]), "x": rng.choice(["f16", "bf16"]), "spare": rng.choice([0, 0, 3])}
    if op == "store":
        case["seqs"] = _log_int(rng, 1, 64)
        case["most"] = _log_int(rng, 1, max(1, MOST_STORE // 2 // (case["hk"] * d * case["seqs"])))
        case["longest"] = case["most"] + _log_int(rng, 1, min(4096, max(1, MOST_READ // (case["hk"] * d * case["seqs"]))))
    elif op == "read":
        case["x"] = rng.choice(["f16", "bf16", "f32"])
        case["seqs"] = _log_int(rng, 1, 64)
        case["longest"] = _log_int(rng, 1, max(1, MOST_READ // 2 // (case["hk"] * d * case["seqs"])))
    else:
        case["hq"] = case["hk"] * rng.choice([1, 2, 4, 5, 8])
        case["seqs"] = _log_int(rng, 1, 128)
        case["longest"] = _log_int(rng, 1, min(200000, max(1, MOST_ATTENTION // 2 // (case["hk"] * d * case["seqs"]))))
        case["most"] = rng.choice([1, 1, rng.randint(2, 8)])
        case["window"] = _log_int(rng, 1, 4096) if rng.random() < 0.3 else 0
        case["causal"] = case["window"] > 0 or rng.random() < 0.8
    return case


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _randint(g, lo, hi, *shape):
    return torch.randint(lo, hi, shape, generator=g, device="cuda")


def _frequencies(case):
    """Angle of each pair for one step of position, and the factor of the rotated part."""
    rot, base = case["rot"], case["base"]
    i = torch.arange(rot // 2, dtype=torch.float64, device="cuda")
    f = base ** (-2.0 * i / rot)
    factor, original = 8.0, 8192.0
    if case["scaling"] == "none":
        return f, 1.0
    if case["scaling"] == "linear":
        return f / factor, 1.0
    if case["scaling"] == "bands":  # the slow pairs stretched, the fast ones kept
        t = ((original * f / (2 * math.pi) - 1.0) / (4.0 - 1.0)).clamp(0.0, 1.0)
        return f * (t + (1.0 - t) / factor), 1.0
    lo, hi = (rot * math.log(original / (turns * 2 * math.pi)) / (2 * math.log(base)) for turns in (32.0, 1.0))
    lo, hi = max(math.floor(lo), 0), min(math.ceil(hi), rot - 1)
    t = ((i - lo) / max(hi - lo, 0.001)).clamp(0.0, 1.0)
    return f * (1.0 - t) + f / factor * t, 0.1 * math.log(factor) + 1.0


def _lengths(case, g):
    """Lengths of the sequences and how many of each one's last tokens take part."""
    seqs, longest, op = case["seqs"], case["longest"], case["op"]
    if not case["ragged"]:
        lengths = torch.full((seqs,), longest, device="cuda")
        counts = lengths.clone() if op == "read" else torch.full((seqs,), min(case["most"], longest), device="cuda")
        return lengths, counts
    # how many rows there are goes by the case alone, as a program's buffers do
    fixed = _gen(1000 * seqs + longest)
    lengths = _randint(fixed if op == "read" else g, (longest + 3) // 4, longest + 1, seqs)
    counts = lengths.clone() if op == "read" else _randint(fixed, 1, min(case["most"], longest) + 1, seqs)
    counts[0] = longest if op == "read" else min(case["most"], longest)
    lengths = torch.maximum(lengths, counts)
    lengths[0] = longest
    if seqs >= 4:  # one that has no tokens yet; in attention it has a row, which sees nothing
        lengths[seqs // 2] = 0
        counts[seqs // 2] = 1 if op == "attention" else 0
    return lengths, counts


def _quantised_rows(s, g):
    """A cache whose pages hold codes and scales of normally distributed rows."""
    case = s["case"]
    pages, hk, page, d, group = s["pages"], case["hk"], case["page"], case["d"], case["group"]
    words, groups = -(-d // 32) * 4, -(-d // group)
    for name in ("k", "v"):
        codes = (_randn(g, pages, hk, page, d) * 2.6).add_(7.5).round_().clamp_(0.0, 15.0).to(torch.uint8)
        codes = torch.nn.functional.pad(codes, (0, 8 * words - d))
        s[name + "_codes"] = (codes[..., 0::2] | (codes[..., 1::2] << 4)).contiguous().view(torch.int32)
        del codes
        scales = torch.exp(0.3 * _randn(g, pages, hk, page, groups)) * 0.33
        lows = scales * (0.8 * _randn(g, pages, hk, page, groups) - 7.5)
        s[name + "_scales"] = torch.stack((scales, lows), -1).half()


def prepare(case, seed):
    g = _gen(seed)
    s = {"case": case}
    dt = DTYPES[case["x"]]
    if case["op"] == "rope":
        tokens, hq, hk, d = case["tokens"], case["hq"], case["hk"], case["d"]
        # queries, keys and values of a token lie together, as their common projection leaves them
        rows = _randn(g, tokens, hq + 2 * hk, d)
        rows[:, :, :: max(1, d // 5)] *= 4.0
        s["rows"] = rows.to(dt)
        s["q"], s["k"] = s["rows"][:, :hq], s["rows"][:, hq:hq + hk]
        s["positions"] = _randint(g, 0, case["far"], 1) + torch.arange(tokens, device="cuda")
        s["q_norm"] = (1.0 + 0.2 * _randn(g, d)).to(dt) if case["norm"] else None
        s["k_norm"] = (1.0 + 0.2 * _randn(g, d)).to(dt) if case["norm"] else None
        s["out"] = [torch.empty((tokens, h, d), dtype=dt, device="cuda") for h in (hq, hk)]
        if own:  # the table of a model's angles, which a program keeps
            from paper_2609_11687_gb300 import kashin as kd
            scaling = None if case["scaling"] == "none" else kd.Scaling(case["scaling"], 8.0, original=8192)
            s["rotation"] = kd.Rotation(case["rot"], case["base"], case["layout"], scaling)
        return s
    seqs, page, hk, d = case["seqs"], case["page"], case["hk"], case["d"]
    lengths, counts = _lengths(case, g)
    starts = torch.zeros(seqs + 1, dtype=torch.int64, device="cuda")
    starts[1:] = counts.cumsum(0)
    s["lengths"], s["starts"] = lengths.int(), starts.int()
    s["most"] = case["longest"] if case["op"] == "read" else min(case["most"], case["longest"])
    s["tokens"] = int(starts[-1]) + case["spare"]
    wide = -(-case["longest"] // page)
    s["pages"] = seqs * wide + 3
    s["table"] = torch.randperm(s["pages"], generator=g, device="cuda")[:seqs * wide].view(seqs, wide).int()
    _quantised_rows(s, g)
    if case["op"] == "store":
        for name in ("k", "v"):
            rows = _randn(g, s["tokens"], hk, d)
            rows[:, :, :: max(1, d // 3)] *= 5.0
            s[name] = rows.to(dt)
    if case["op"] == "attention":
        s["q"] = (_randn(g, s["tokens"], case["hq"], d) * 1.5 * math.sqrt(128 / max(d, 64))).to(dt)
        s["lse"] = torch.full((s["tokens"], case["hq"]), -math.inf, device="cuda")
        s["out"] = torch.zeros((s["tokens"], case["hq"], d), dtype=dt, device="cuda")
    else:
        s["out"] = [torch.zeros((s["tokens"], hk, d), dtype=dt, device="cuda") for _ in range(2)]
    if own:  # the handles that a program keeps: the cache, and one step's sequences
        from paper_2609_11687_gb300 import kashin as kd
        s["cache"] = kd.Cache4(s["k_codes"], s["k_scales"], s["v_codes"], s["v_scales"], d=d, group=case["group"])
        s["sequences"] = kd.Sequences(s["table"], s["lengths"], s["starts"] if case["ragged"] or case["spare"] else None,
                                      most=s["most"], longest=case["longest"])
    return s


def _plain_rotate(x, weight, cos, sin, layout, rot):
    x = x.float()
    if weight is not None:
        x = x * torch.rsqrt((x * x).mean(2, keepdim=True) + 1e-6) * weight.float()
    r, rest = x[:, :, :rot], x[:, :, rot:]
    a, b = (r[:, :, :rot // 2], r[:, :, rot // 2:]) if layout == "half" else (r[:, :, 0::2], r[:, :, 1::2])
    a, b = a * cos - b * sin, b * cos + a * sin
    r = torch.cat((a, b), 2) if layout == "half" else torch.stack((a, b), 3).flatten(2)
    return torch.cat((r, rest), 2)


def _plain_rope(s):
    case = s["case"]
    f, amplitude = _frequencies(case)
    angle = s["positions"].double()[:, None, None] * f
    cos, sin = (amplitude * torch.cos(angle)).float(), (amplitude * torch.sin(angle)).float()
    q = _plain_rotate(s["q"], s["q_norm"], cos, sin, case["layout"], case["rot"]).to(s["q"].dtype)
    k = _plain_rotate(s["k"], s["k_norm"], cos, sin, case["layout"], case["rot"]).to(s["k"].dtype)
    return {"q": q, "k": k}


def _places(s):
    """Of each row its sequence, its position there (-1: none) and its page and place in that."""
    row = torch.arange(s["tokens"], device="cuda")
    starts, page = s["starts"].long(), s["case"]["page"]
    seq = (torch.searchsorted(starts, row, right=True) - 1).clamp(max=s["case"]["seqs"] - 1)
    at = s["lengths"].long()[seq] - (starts[seq + 1] - row)
    at = torch.where(row < starts[-1], at, torch.full_like(at, -1))
    safe = at.clamp(min=0)
    return seq, at, s["table"].long()[seq, safe // page], safe % page


def _beside(h, by):
    """The fp16 value next to each of ``h``, above (by = 1) or below (by = -1)."""
    bits = h.view(torch.int16).int()
    order = torch.where(bits < 0, -(bits & 0x7FFF), bits) + by
    return torch.where(order < 0, order.abs() - 0x8000, order).to(torch.int16).view(torch.float16)


def _plain_quantise(x, group, words):
    """4-bit codes of each group of a row with its scale (rounded up) and lowest value (down)."""
    x = x.float()
    d = x.shape[-1]
    groups = -(-d // group)
    short = groups * group - d
    padded = torch.cat((x, x[..., -1:].expand(*x.shape[:-1], short)), -1).view(*x.shape[:-1], groups, group)
    lo, hi = padded.amin(-1), padded.amax(-1)
    low = lo.half()
    low = torch.where(low.float() > lo, _beside(low, -1), low)
    scale = (hi - low.float()) / torch.full_like(hi, 15.0)
    up = scale.half()
    up = torch.where(up.float() < scale, _beside(up, 1), up)
    step = torch.where(up == 0, torch.ones_like(up), up).float()[..., None]
    codes = ((padded - low.float()[..., None]) / step).round().clamp(0.0, 15.0).to(torch.int32).flatten(-2)[..., :d]
    codes = torch.nn.functional.pad(codes, (0, 8 * words - d)).view(*x.shape[:-1], words, 8)
    packed = (codes << torch.arange(0, 32, 4, device="cuda", dtype=torch.int32)).sum(-1, dtype=torch.int32)
    return packed, torch.stack((up, low), -1)


def _plain_values(codes, scales, group, d):
    c = (codes[..., None] >> torch.arange(0, 32, 4, device="cuda", dtype=torch.int32)) & 15
    c = c.flatten(-2)[..., :d].float()
    c *= scales[..., 0].float().repeat_interleave(group, -1)[..., :d]
    c += scales[..., 1].float().repeat_interleave(group, -1)[..., :d]
    return c


def _plain_read(s):
    case = s["case"]
    _, at, page, place = _places(s)
    out = {}
    for name in ("k", "v"):
        x = _plain_values(s[name + "_codes"][page, :, place], s[name + "_scales"][page, :, place], case["group"], case["d"])
        out[name] = (x * (at >= 0)[:, None, None]).to(DTYPES[case["x"]])
    return out


def _plain_store(s):
    case = s["case"]
    _, at, page, place = _places(s)
    page, place = page[at >= 0], place[at >= 0]
    for name in ("k", "v"):
        codes, scales = _plain_quantise(s[name][at >= 0], case["group"], s[name + "_codes"].shape[-1])
        s[name + "_codes"][page, :, place] = codes
        s[name + "_scales"][page, :, place] = scales
    return _plain_read(s)


def _plain_attention(s):
    case = s["case"]
    hq, hk, d, window, most = case["hq"], case["hk"], case["d"], case["window"], s["most"]
    lengths, table = s["lengths"].long(), s["table"].long()

    def dense(name):  # (sequences, key heads, places, d)
        x = _plain_values(s[name + "_codes"][table], s[name + "_scales"][table], case["group"], d)
        return x.transpose(1, 2).flatten(2, 3)

    # the rows of each sequence, laid out (sequence, row)
    seq, at, _, _ = _places(s)
    row = torch.arange(s["tokens"], device="cuda")
    nth = row - s["starts"].long()[seq]
    real = row < s["starts"][-1]
    q = torch.zeros((case["seqs"], most, hq, d), device="cuda")
    position = torch.full((case["seqs"], most), -1, device="cuda")
    q[seq[real], nth[real]] = s["q"].float()[real]
    position[seq[real], nth[real]] = at[real]
    q = q.transpose(1, 2).reshape(case["seqs"], hk, hq // hk * most, d)
    k = dense("k")
    score = q @ k.transpose(2, 3) * (d ** -0.5)
    del k
    key = torch.arange(score.shape[3], device="cuda")
    seen = (key < lengths[:, None])[:, None, :].expand(-1, most, -1)
    if case["causal"]:
        seen = seen & (key <= position[:, :, None])
        if window:
            seen = seen & (key > position[:, :, None] - window)
    seen = seen.repeat(1, hq // hk, 1)[:, None]
    score = torch.where(seen, score, torch.full_like(score, -math.inf))
    top = score.amax(3, keepdim=True)
    empty = top == -math.inf
    p = torch.exp(score - torch.where(empty, torch.zeros_like(top), top))
    del score
    total = p.sum(3, keepdim=True)
    v = dense("v")
    y = (p @ torch.where((key < lengths[:, None])[:, None, :, None], v, torch.zeros_like(v))) / torch.where(empty, torch.ones_like(total), total)
    lse = torch.where(empty, top, top + torch.log(total))
    y = y.view(case["seqs"], hq, most, d).transpose(1, 2)
    lse = lse.view(case["seqs"], hq, most).transpose(1, 2)
    nth = nth.clamp(0, most - 1)
    return {"out": torch.where(real[:, None, None], y[seq, nth], torch.zeros_like(y[seq, nth])).to(s["q"].dtype),
            "lse": torch.where(real[:, None], lse[seq, nth], torch.full_like(lse[seq, nth], -math.inf))}


def run(state):
    case = state["case"]
    op = case["op"]
    if not own:
        return {"rope": _plain_rope, "store": _plain_store, "read": _plain_read, "attention": _plain_attention}[op](state)
    from paper_2609_11687_gb300 import kashin as kd
    if op == "rope":
        q, k = kd.rope(state["q"], state["k"], state["positions"], state["rotation"], q_norm=state["q_norm"], k_norm=state["k_norm"],
                       eps=1e-6, out=state["out"])
        return {"q": q, "k": k}
    if op == "attention":
        out = kd.attention_4bit(state["cache"], state["q"], state["sequences"], causal=case["causal"], window=case["window"],
                                out=state["out"], lse=state["lse"])
        return {"out": out, "lse": state["lse"]}
    if op == "store":
        kd.cache_write_4bit(state["cache"], state["k"], state["v"], state["sequences"])
    k, v = kd.cache_read_4bit(state["cache"], state["sequences"], out=state["out"])
    return {"k": k, "v": v}


def _shares(case):
    """Expected tokens of the sequences, and rows that take part."""
    seqs, longest = case["seqs"], case["longest"]
    most = longest if case["op"] == "read" else min(case["most"], longest)
    if not case["ragged"]:
        return seqs * longest, seqs * most
    held = longest + (seqs - 1 - (seqs >= 4)) * 0.625 * longest
    return held, held if case["op"] == "read" else most + (seqs - 1) * (most + 1) / 2


def work(case):
    if case["op"] == "rope":
        values = case["tokens"] * (case["hq"] + case["hk"]) * case["d"]
        return {"bytes": 2 * values * BYTES[case["x"]] + 8 * case["tokens"], "flops": (10 if case["norm"] else 6) * values}
    d, hk = case["d"], case["hk"]
    held, rows = _shares(case)
    row = 2 * hk * (d / 2 + 4 * -(-d // case["group"]))  # of a token's key and value in the cache
    if case["op"] == "store":
        return {"bytes": rows * (2 * 2 * hk * d * BYTES[case["x"]] + 2 * row), "flops": 8 * rows * hk * d}
    if case["op"] == "read":
        return {"bytes": rows * (row + 2 * hk * d * BYTES[case["x"]]), "flops": 4 * rows * hk * d}
    if case["window"]:
        held = min(held, case["seqs"] * (case["window"] + min(case["most"], case["longest"])))
    return {"bytes": held * row + rows * case["hq"] * (2 * d * BYTES[case["x"]] + 4),
            "flops": 4 * held * (rows / case["seqs"]) * case["hq"] * d}


def _exact_values(codes, scales, group, d):
    """Values of codes (..., words) with scales (..., groups, 2), one channel after the other."""
    channel = torch.arange(d, device="cuda")
    c = codes[..., channel // 8].long() & 0xFFFFFFFF
    c = (c >> (4 * (channel % 8))) % 16
    which = channel // group
    return c.double() * scales[..., which, 0].double() + scales[..., which, 1].double()


def _exact_code_values(x, group):
    """What rows are held as: each group from its lowest value (fp16, rounded down) in 15 steps
    (fp16, rounded up)."""
    out = torch.empty_like(x)
    for a in range(0, x.shape[-1], group):
        part = x[..., a:a + group]
        lo, hi = part.min(-1, keepdim=True).values, part.max(-1, keepdim=True).values

        def to_half(v, down):
            v = v.cpu().numpy()
            h = v.astype(np.float16)
            wrong = h.astype(np.float64) > v if down else h.astype(np.float64) < v
            h = np.where(wrong, np.nextafter(h, np.float16(-np.inf if down else np.inf)), h)
            return torch.from_numpy(h.astype(np.float64)).cuda()

        low = to_half(lo, True)
        step = to_half((hi - low) / 15.0, False)
        code = torch.where(step > 0, (part - low) / torch.where(step > 0, step, torch.ones_like(step)), torch.zeros_like(part))
        out[..., a:a + group] = low + step * code.round()
    return out


def exact(case, seed):
    """The definitions in 64 bits."""
    s = prepare(case, seed)
    f64 = torch.float64
    if case["op"] == "rope":
        f, amplitude = _frequencies(case)
        out, rot = {}, case["rot"]
        turn = torch.polar(torch.full((case["tokens"], rot // 2), amplitude, dtype=f64, device="cuda"), torch.outer(s["positions"].to(f64), f))
        for name in ("q", "k"):
            x = s[name].to(f64)
            if s[name + "_norm"] is not None:
                x = x / (x.square().sum(2, keepdim=True) / case["d"] + 1e-6).sqrt() * s[name + "_norm"].to(f64)
            pair = x[..., :rot].unflatten(2, (2, rot // 2)).transpose(2, 3) if case["layout"] == "half" else x[..., :rot].unflatten(2, (rot // 2, 2))
            pair = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * turn[:, None])
            y = x.clone()
            y[..., :rot] = (pair.transpose(2, 3) if case["layout"] == "half" else pair).flatten(2)
            out[name] = y
        return out
    page, d, group = case["page"], case["d"], case["group"]
    starts, lengths = s["starts"].tolist(), s["lengths"].tolist()
    if case["op"] in ("store", "read"):
        out = {name: torch.zeros((s["tokens"], case["hk"], d), dtype=f64, device="cuda") for name in ("k", "v")}
        for i in range(case["seqs"]):
            n = starts[i + 1] - starts[i]
            at = torch.arange(lengths[i] - n, lengths[i], device="cuda")
            for name in ("k", "v"):
                if case["op"] == "store":
                    x = _exact_code_values(s[name][starts[i]:starts[i + 1]].to(f64), group)
                else:
                    p = s["table"][i].long()[at // page]
                    x = _exact_values(s[name + "_codes"][p, :, at % page], s[name + "_scales"][p, :, at % page], group, d)
                out[name][starts[i]:starts[i + 1]] = x
        return out
    hq, hk = case["hq"], case["hk"]
    y = torch.zeros((s["tokens"], hq, d), dtype=f64, device="cuda")
    lse = torch.full((s["tokens"], hq), -math.inf, dtype=f64, device="cuda")
    for i in range(case["seqs"]):
        n, length = starts[i + 1] - starts[i], lengths[i]
        if n == 0 or length == 0:
            continue
        at = torch.arange(length, device="cuda")
        p = s["table"][i].long()[at // page]
        where = torch.arange(length - n, length, device="cuda")[:, None]
        hidden = torch.zeros((n, length), dtype=torch.bool, device="cuda")
        if case["causal"]:
            hidden = at > where
            if case["window"]:
                hidden |= at <= where - case["window"]
        for h in range(hk):
            k = _exact_values(s["k_codes"][p, h, at % page], s["k_scales"][p, h, at % page], group, d)
            v = _exact_values(s["v_codes"][p, h, at % page], s["v_scales"][p, h, at % page], group, d)
            heads = slice(h * (hq // hk), (h + 1) * (hq // hk))
            q = s["q"][starts[i]:starts[i + 1], heads].to(f64)
            score = torch.einsum("thd,ld->thl", q, k) / math.sqrt(d)
            score.masked_fill_(hidden[:, None, :], -math.inf)
            total = torch.logsumexp(score, 2)
            lse[starts[i]:starts[i + 1], heads] = total
            # where a row sees nothing its sum is empty
            y[starts[i]:starts[i + 1], heads] = torch.einsum("thl,ld->thd", torch.nan_to_num((score - total[..., None]).exp(), nan=0.0), v)
    return {"out": y, "lse": lse}
