"""Cases of the operators around a tied embedding / pre-softmax projection weight [vocab, d].

  embed    rows of the table on the way in: lookup, scale, position rows, dropout; and the value rows that the
           embedding's gradient brings to the densify
  dropout  dropout of a sub-layer's output added to the residual stream, and its gradient
  project  the table on the way out: logits = x W^T with both operands in 8-bit floating point, one scale for each
           block of 128; `step` adds the quantisation of the changed weight and both gradients
  sample   a token per row of logits, from given uniform numbers, with temperature, top-k, top-p and min-p

The plain forms below define the arithmetic.  Random bits of dropout: Philox4x32-10 (Salmon et al., "Parallel random
numbers: as easy as 1, 2, 3", 2011), key = the 64-bit seed, counter = (column / 8, row, offset low, offset high); the
eight 16-bit halves of its four words, low half first, belong to eight consecutive columns of the row.
"""
import math

import numpy as np
import torch

own = False

VOCAB = 33708           # shared sub-word vocabulary of the tied weight
E4M3_MAX = 448.0        # largest finite value of the 8-bit type
LOW32 = 0xFFFFFFFF
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # the smallest training case of this repository: latency of one call each way
        {"name": "embed tiny", "op": "embed", "rows": 512, "d": 64, "vocab": 1000, "weight": "f32", "out": "f32", "index": "i64", "positions": 64, "p": 0.1},
        # encoder and decoder lookups of a base-size step, fp32 master weight, bf16 activations
        {"name": "embed base", "op": "embed", "rows": 8192, "d": 512, "vocab": VOCAB, "weight": "f32", "out": "bf16", "index": "i64", "positions": 256, "p": 0.1},
        # the same for a big-size step
        {"name": "embed big", "op": "embed", "rows": 25600, "d": 1024, "vocab": VOCAB, "weight": "bf16", "out": "bf16", "index": "i32", "positions": 1024, "p": 0.3},
        # a sub-layer's output of a base-size step
        {"name": "dropout base", "op": "dropout", "rows": 8192, "d": 512, "x": "bf16", "out": "bf16", "residual": True, "pad": 0, "p": 0.1},
        # odd rows, not aligned, in a wider buffer
        {"name": "dropout odd", "op": "dropout", "rows": 12801, "d": 1021, "x": "f32", "out": "f32", "residual": True, "pad": 3, "p": 0.25},
        # one token being generated
        {"name": "project one token", "op": "project", "step": False, "tokens": 1, "d": 1024, "vocab": VOCAB, "x": "bf16", "out": "f32"},
        # a beam search's or a small batch's tokens being generated
        {"name": "project batch", "op": "project", "step": False, "tokens": 48, "d": 512, "vocab": VOCAB, "x": "bf16", "out": "bf16"},
        # scoring of a validation batch
        {"name": "project scoring", "op": "project", "step": False, "tokens": 4096, "d": 1024, "vocab": VOCAB, "x": "bf16", "out": "bf16"},
        # a training step's share of the projection, base size
        {"name": "project step base", "op": "project", "step": True, "tokens": 4096, "d": 512, "vocab": VOCAB, "x": "bf16", "out": "bf16"},
        # the same, big size, tokens that fill no tile
        {"name": "project step big", "op": "project", "step": True, "tokens": 8111, "d": 1024, "vocab": VOCAB, "x": "bf16", "out": "bf16"},
        # one request being answered
        {"name": "sample one row", "op": "sample", "rows": 1, "vocab": VOCAB, "x": "f32", "top_k": True, "top_p": True, "min_p": False},
        # a large batch of requests, each with settings of its own
        {"name": "sample batch", "op": "sample", "rows": 512, "vocab": 65536, "x": "bf16", "top_k": True, "top_p": True, "min_p": True},
    ]


def _between(rng, low, high):
    """A whole number, spread evenly over the logarithm."""
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 1)))))))


def draw(rng):
    op = rng.choice(["embed", "dropout", "project", "sample"])
    if op == "embed":
        return {"op": op, "rows": _between(rng, 1, 25600), "d": rng.choice([64, 512, 1024, 8 * rng.randint(8, 128), rng.randint(33, 1024)]), "vocab": rng.choice([1000, VOCAB, 65536]),
                "weight": rng.choice(["f32", "bf16"]), "out": rng.choice(["f32", "bf16"]), "index": rng.choice(["i32", "i64"]), "positions": rng.choice([0, rng.randint(1, 1024)]), "p": rng.choice([0.0, 0.1, 0.3])}
    if op == "dropout":
        return {"op": op, "rows": _between(rng, 1, 25600), "d": rng.choice([64, 512, 1024, rng.randint(33, 1024)]), "x": rng.choice(["f32", "bf16"]),
                "out": rng.choice(["f32", "bf16"]), "residual": rng.choice([True, False]), "pad": rng.choice([0, 0, 8, rng.randint(1, 63)]), "p": rng.choice([0.1, 0.2, 0.5])}
    if op == "project":
        step, out = rng.choice([True, False]), rng.choice(["f32", "bf16"])
        return {"op": op, "step": step, "tokens": _between(rng, 16 if step else 1, 4000 if out == "f32" else 8000), "d": rng.choice([512, 1024, rng.randint(64, 1024)]), "vocab": rng.choice([1000, VOCAB, rng.randint(1000, VOCAB)]),
                "x": rng.choice(["f32", "bf16"]), "out": out}
    return {"op": op, "rows": _between(rng, 1, 512), "vocab": rng.choice([1000, VOCAB, 65536, rng.randint(500, 65536)]), "x": rng.choice(["f32", "bf16"]),
            "top_k": rng.choice([True, False]), "top_p": rng.choice([True, False]), "min_p": rng.choice([True, False])}


# ---- inputs ------------------------------------------------------------------------------------------------------
def _zipf(n, vocab, g):
    """Token ids that follow a bounded Zipf law with exponent 1.1."""
    cdf = torch.arange(1, vocab + 1, device="cuda", dtype=torch.float64).pow(-1.1).cumsum(0)
    return torch.searchsorted(cdf, torch.rand(n, device="cuda", dtype=torch.float64, generator=g) * cdf[-1]).clamp_(max=vocab - 1)


def _padded(rows, d, pad, dtype, g):
    """A [rows, d] tensor inside rows of d + pad elements."""
    return torch.randn(rows, d + pad, device="cuda", generator=g).to(dtype)[:, :d]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": case, "seed": (seed * 0x9E3779B97F4A7C15 + 12345) & 0x7FFFFFFFFFFFFFFF, "offset": 7 + (seed << 33) % (1 << 50)}
    op = case["op"]
    if op == "embed":
        n, d, vocab = case["rows"], case["d"], case["vocab"]
        s["indices"] = _zipf(n, vocab, g).to(torch.int32 if case["index"] == "i32" else torch.int64)
        s["weight"] = (torch.randn(vocab, d, device="cuda", generator=g) * d ** -0.5).to(TYPES[case["weight"]])
        s["position"] = torch.sin(torch.rand(case["positions"], d, device="cuda", generator=g) * 100) if case["positions"] else None
        s["grad"] = (torch.randn(n, d, device="cuda", generator=g) * 0.02).to(TYPES[case["out"]])
        s["scale"] = d ** 0.5
        s["out"] = torch.empty(n, d, device="cuda", dtype=TYPES[case["out"]])
        s["values"] = torch.empty(n, d, device="cuda", dtype=TYPES[case["weight"]])
    elif op == "dropout":
        n, d, pad = case["rows"], case["d"], case["pad"]
        s["x"] = _padded(n, d, pad, TYPES[case["x"]], g)
        s["residual"] = _padded(n, d, pad, TYPES[case["out"]], g) if case["residual"] else None
        s["grad"] = _padded(n, d, pad, TYPES[case["out"]], g)
        s["out"] = torch.empty(n, d, device="cuda", dtype=TYPES[case["out"]])
        s["dx"] = torch.empty(n, d, device="cuda", dtype=TYPES[case["x"]])
    elif op == "project":
        m, d, vocab = case["tokens"], case["d"], case["vocab"]
        s["x"] = torch.randn(m, d, device="cuda", generator=g).to(TYPES[case["x"]])
        s["weight"] = torch.randn(vocab, d, device="cuda", generator=g) * d ** -0.5
        s["logits"] = torch.empty(m, vocab, device="cuda", dtype=TYPES[case["out"]])
        if case["step"]:
            prob = torch.softmax(torch.randn(m, vocab, device="cuda", generator=g) * 2, -1)
            prob[torch.arange(m, device="cuda"), _zipf(m, vocab, g)] -= 1
            s["dlogits"] = (prob / m).to(TYPES[case["out"]])
            s["dx"] = torch.empty(m, d, device="cuda", dtype=TYPES[case["x"]])
            s["dweight"] = torch.empty(vocab, d, device="cuda")
        else:  # the weight stays as it is between calls: its 8-bit form is kept
            s["q"], s["q_scale"] = _square(s["weight"])
        if own:
            import paper_1905_04035_b200 as dst
            s["projection"] = dst.TiedProjection(vocab, d, m, training=case["step"])
            if not case["step"]:
                s["projection"].update(s["weight"])
    else:
        n, vocab = case["rows"], case["vocab"]
        unigram = -1.1 * torch.log(torch.arange(1, vocab + 1, device="cuda", dtype=torch.float32))
        s["logits"] = (torch.randn(n, vocab, device="cuda", generator=g) * 2 + unigram[torch.randperm(vocab, device="cuda", generator=g)] + 12).to(TYPES[case["x"]])
        s["uniform"] = torch.rand(n, device="cuda", generator=g)
        s["temperature"] = 0.5 + torch.rand(n, device="cuda", generator=g)
        s["top_k"] = torch.randint(1, 200, (n,), device="cuda", generator=g, dtype=torch.int32) if case["top_k"] else None
        s["top_p"] = 0.7 + 0.3 * torch.rand(n, device="cuda", generator=g) if case["top_p"] else None
        s["min_p"] = 0.1 * torch.rand(n, device="cuda", generator=g) if case["min_p"] else None
        s["tokens"] = torch.empty(n, device="cuda", dtype=torch.int64)
        s["prob"] = torch.empty(n, device="cuda")
    return s


# ---- plain forms -------------------------------------------------------------------------------------------------
def _halves(n, d, seed, offset):
    """The 16-bit number of every element of [n, d]."""
    c0 = torch.arange(-(-d // 8), device="cuda").view(1, -1).expand(n, -1)
    c1 = torch.arange(n, device="cuda").view(-1, 1).expand(-1, c0.shape[1])
    c2, c3 = torch.full_like(c0, offset & LOW32), torch.full_like(c0, offset >> 32)
    k0, k1 = seed & LOW32, seed >> 32
    for _ in range(10):  # the generator's ten rounds
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((p1 >> 32) & LOW32) ^ c1 ^ k0, p1 & LOW32, ((p0 >> 32) & LOW32) ^ c3 ^ k1, p0 & LOW32
        k0, k1 = (k0 + 0x9E3779B9) & LOW32, (k1 + 0xBB67AE85) & LOW32
    words = torch.stack([c0, c1, c2, c3], -1)
    return torch.stack([words & 0xFFFF, words >> 16], -1).reshape(n, -1)[:, :d]


def _factor(n, d, p, seed, offset):
    """1 / (1 - p) where the element is kept and 0 where it is dropped; p is rounded to a multiple of 2^-16."""
    cut = round(p * 65536)
    if cut == 0:
        return torch.ones(n, d, device="cuda")
    return (_halves(n, d, seed, offset) >= cut).float() * (65536 / (65536 - cut))


def _power(amax):
    """The smallest power of two that brings amax to at most 448."""
    mantissa, exponent = torch.frexp(amax.clamp_min(2.0 ** -100))
    return torch.ldexp(torch.ones_like(amax), exponent - 9 + (mantissa > 0.875).int())


def _blocks(x):
    rows, cols = x.shape
    return torch.nn.functional.pad(x.float(), (0, -cols % 128)).view(rows, -1, 128)


def _rounded_rows(x):
    """x as its 8-bit form stands for it: one scale for every 128 consecutive elements of a row."""
    b = _blocks(x)
    scale = _power(b.abs().amax(-1, keepdim=True))
    return ((b / scale).to(torch.float8_e4m3fn).float() * scale).reshape(x.shape[0], -1)[:, :x.shape[1]]


def _square(w):
    """8-bit form of w with one scale for every 128 x 128 block."""
    rows, cols = w.shape
    b = torch.nn.functional.pad(w.float(), (0, -cols % 128, 0, -rows % 128))
    b = b.view(b.shape[0] // 128, 128, -1, 128)
    scale = _power(b.abs().amax((1, 3), keepdim=True))
    return (b / scale).to(torch.float8_e4m3fn), scale


def _of_square(q, scale, shape):
    b = q.float() * scale
    return b.reshape(b.shape[0] * 128, -1)[:shape[0], :shape[1]]


def _share(part, total):
    """floor(part / 2^24 * total) of whole numbers, without passing 64 bits."""
    return part * (total >> 24) + ((part * (total & 0xFFFFFF)) >> 24)


def _sample(s):
    x = s["logits"].float()
    n, vocab = x.shape
    x = torch.where(torch.isnan(x), torch.full_like(x, -math.inf), x)
    top = x.amax(-1, keepdim=True)
    z = torch.where(x == top, torch.zeros_like(x), (x - top) * (1 / s["temperature"]).view(-1, 1))
    e = torch.exp(z)
    weight = torch.round(e * 2.0 ** 31).long()  # whole numbers: their sums have no order
    _, order = torch.sort(x, dim=-1, descending=True, stable=True)
    ranked = weight.gather(-1, order)
    keep = torch.ones_like(order, dtype=torch.bool)
    if s["top_k"] is not None:
        keep &= torch.arange(vocab, device="cuda") < s["top_k"].view(-1, 1)
    if s["top_p"] is not None:
        mass = ranked * keep
        upto = _share((s["top_p"] * 2.0 ** 24).long().view(-1, 1), mass.sum(-1, keepdim=True)).clamp_min(1)
        keep &= mass.cumsum(-1) - mass < upto
    if s["min_p"] is not None:
        keep &= e.gather(-1, order) >= s["min_p"].view(-1, 1)
    kept = weight * torch.zeros_like(keep).scatter_(-1, order, keep)
    upto = kept.cumsum(-1)
    at = _share((s["uniform"] * 2.0 ** 24).long().view(-1, 1), upto[:, -1:])
    token = (upto > at).int().argmax(-1, keepdim=True)
    return {"tokens": token.view(-1), "prob": (kept.gather(-1, token).float() / upto[:, -1:].float()).view(-1)}


def run(s):
    c, op = s["case"], s["case"]["op"]
    if own:
        import paper_1905_04035_b200 as dst
        if op == "embed":
            dst.dst_embed(s["indices"], s["weight"], s["out"], scale=s["scale"], position=s["position"], p=c["p"], seed=s["seed"], offset=s["offset"])
            dst.dst_dropout(s["grad"], s["values"], c["p"], s["seed"], s["offset"], scale=s["scale"])
            return {"out": s["out"], "values": s["values"]}
        if op == "dropout":
            dst.dst_dropout(s["x"], s["out"], c["p"], s["seed"], s["offset"], residual=s["residual"])
            dst.dst_dropout(s["grad"], s["dx"], c["p"], s["seed"], s["offset"])
            return {"out": s["out"], "dx": s["dx"]}
        if op == "project":
            if not c["step"]:
                return {"logits": s["projection"].logits(s["x"], s["logits"])}
            s["projection"].update(s["weight"])
            s["projection"].logits(s["x"], s["logits"])
            s["projection"].backward(s["dlogits"], s["x"], s["dx"], s["dweight"])
            return {"logits": s["logits"], "dx": s["dx"], "dweight": s["dweight"]}
        dst.dst_sample(s["logits"], s["uniform"], s["tokens"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"], prob=s["prob"])
        return {"tokens": s["tokens"], "prob": s["prob"]}
    if op == "embed":
        n, d = c["rows"], c["d"]
        factor = _factor(n, d, c["p"], s["seed"], s["offset"])
        rows = s["weight"][s["indices"].long()].float() * s["scale"]
        if s["position"] is not None:
            rows = rows + s["position"][torch.arange(n, device="cuda") % c["positions"]]
        return {"out": (rows * factor).to(s["out"].dtype), "values": (s["grad"].float() * factor * s["scale"]).to(s["values"].dtype)}
    if op == "dropout":
        factor = _factor(c["rows"], c["d"], c["p"], s["seed"], s["offset"])
        out = s["x"].float() * factor
        if s["residual"] is not None:
            out = out + s["residual"].float()
        return {"out": out.to(s["out"].dtype), "dx": (s["grad"].float() * factor).to(s["dx"].dtype)}
    if op == "project":
        x = s["x"]
        q, scale = _square(s["weight"]) if c["step"] else (s["q"], s["q_scale"])
        w = _of_square(q, scale, (c["vocab"], c["d"]))
        logits = (_rounded_rows(x) @ w.T).to(s["logits"].dtype)
        if not c["step"]:
            return {"logits": logits}
        dx = _rounded_rows(s["dlogits"]) @ w
        dw = _rounded_rows(s["dlogits"].T) @ _rounded_rows(x.T).T
        return {"logits": logits, "dx": dx.to(x.dtype), "dweight": dw}
    return _sample(s)


# ---- what a pass cannot do without -------------------------------------------------------------------------------
def work(case):
    size = lambda t: 4 if t == "f32" else 2  # noqa: E731
    op = case["op"]
    if op == "embed":
        n, d = case["rows"], case["d"]
        rows = min(n, case["vocab"]) if n < 512 else min(n, case["vocab"]) // 2  # rows of the table that are read once
        return {"bytes": n * (8 if case["index"] == "i64" else 4) + rows * d * size(case["weight"]) + case["positions"] * d * 4 + n * d * (2 * size(case["out"]) + size(case["weight"])), "flops": 4 * n * d}
    if op == "dropout":
        n = case["rows"] * case["d"]
        return {"bytes": n * (2 * size(case["x"]) + (2 + bool(case["residual"])) * size(case["out"])), "flops": 3 * n}
    if op == "project":
        m, d, vocab, x, out = case["tokens"], case["d"], case["vocab"], size(case["x"]), size(case["out"])
        if not case["step"]:
            return {"bytes": m * d * x + vocab * d + m * vocab * out, "flops": 2 * m * d * vocab}
        return {"bytes": 2 * m * d * x + 2 * vocab * d * 4 + 2 * m * vocab * out, "flops": 6 * m * d * vocab}
    return {"bytes": case["rows"] * (case["vocab"] * size(case["x"]) + 28), "flops": 6 * case["rows"] * case["vocab"]}


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------
def _exact_factor(n, d, p, seed, offset):
    """The dropout factors on the host, from the generator's published round function."""
    cut = int(np.rint(p * 65536))
    groups = -(-d // 8)
    ctr = np.empty((4, n, groups), np.uint64)
    ctr[0], ctr[1], ctr[2], ctr[3] = np.arange(groups)[None], np.arange(n)[:, None], offset % 2 ** 32, offset // 2 ** 32
    key = [seed % 2 ** 32, seed // 2 ** 32]
    low, half = np.uint64(LOW32), np.uint64(32)
    for r in range(10):
        a, b = np.uint64(0xD2511F53) * ctr[0], np.uint64(0xCD9E8D57) * ctr[2]
        ctr = np.stack([(b >> half) ^ ctr[1] ^ np.uint64((key[0] + r * 0x9E3779B9) % 2 ** 32), b & low, (a >> half) ^ ctr[3] ^ np.uint64((key[1] + r * 0xBB67AE85) % 2 ** 32), a & low])
    bits = np.ascontiguousarray(np.moveaxis(ctr, 0, -1).astype("<u4")).view("<u2").reshape(n, groups * 8)[:, :d]
    return torch.from_numpy(np.where(bits >= cut, 65536.0 / (65536 - cut), 0.0)).cuda()


def _exact_codes(x, rows, cols):
    """x in 64 bits, rounded to 8 bits with one power of two for each block of rows x cols elements."""
    x = x.double()
    n, m = x.shape
    full = x.new_zeros(-(-n // rows) * rows, -(-m // cols) * cols)
    full[:n, :m] = x
    b = full.unfold(0, rows, rows).unfold(1, cols, cols)
    unit = torch.exp2(torch.ceil(torch.log2(b.abs().amax((2, 3)).clamp_min(2.0 ** -100) / E4M3_MAX)))
    unit = unit.repeat_interleave(rows, 0).repeat_interleave(cols, 1)[:n, :m]
    v = x / unit
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -6))) - 3)  # three bits after the leading one; 2^-9 below the normal range
    return torch.round(v / step) * step * unit


def _exact_sample(s):
    tokens, probs = [], []
    value = lambda name, row, none: none if s[name] is None else s[name][row].item()  # noqa: E731
    for row in range(s["logits"].shape[0]):
        x = s["logits"][row].double().cpu().numpy()
        e = np.exp((x - x.max()) / s["temperature"][row].item())
        w = np.rint(e * 2.0 ** 31)
        order = np.lexsort((np.arange(len(x)), -x))[: value("top_k", row, len(x))]
        before = np.concatenate([[0.0], np.cumsum(w[order])])
        order = order[before[:-1] < max(1.0, np.floor(min(1.0, value("top_p", row, 1.0)) * before[-1]))]
        order = np.sort(order[e[order] >= value("min_p", row, 0.0)])
        total = np.cumsum(w[order])
        at = int(np.searchsorted(total, np.floor(s["uniform"][row].item() * total[-1]), side="right"))
        tokens.append(int(order[at]))
        probs.append(w[order[at]] / total[-1])
    return {"tokens": torch.tensor(tokens), "prob": torch.tensor(probs, dtype=torch.float64)}


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "embed":
        factor = _exact_factor(case["rows"], case["d"], case["p"], s["seed"], s["offset"])
        rows = s["weight"].double()[s["indices"].long()] * s["scale"]
        if case["positions"]:
            rows += s["position"].double().repeat(-(-case["rows"] // case["positions"]), 1)[:case["rows"]]
        return {"out": rows * factor, "values": s["grad"].double() * s["scale"] * factor}
    if op == "dropout":
        factor = _exact_factor(case["rows"], case["d"], case["p"], s["seed"], s["offset"])
        return {"out": s["x"].double() * factor + (0 if s["residual"] is None else s["residual"].double()), "dx": s["grad"].double() * factor}
    if op == "project":
        w = _exact_codes(s["weight"], 128, 128)
        logits = torch.mm(_exact_codes(s["x"], 1, 128), w.T)
        if not case["step"]:
            return {"logits": logits}
        dx = torch.mm(_exact_codes(s["dlogits"], 1, 128), w)
        dw = torch.mm(_exact_codes(s["dlogits"], 128, 1).T, _exact_codes(s["x"], 128, 1))
        return {"logits": logits, "dx": dx, "dweight": dw}
    return _exact_sample(s)
