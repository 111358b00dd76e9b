"""Cases of more operators around a tied embedding / pre-softmax projection weight [vocab, d].

  logprob   log probabilities of given tokens from a row of logits, with the row's entropy and its most likely tokens
            ("score"); the same with the gradient of a loss that is a weighted sum of them, in one pass ("loss"); and
            forward and gradient apart, with entropy, where the weights come from in between ("policy")
  norm      root-mean-square norm of the residual stream with a sub-layer's output added, and its gradient ("train");
            and the norm before the projection, straight to 8 bits, with the projection ("project")
  clip      global norm of a list of gradients, and the list scaled down to a largest norm
  project4  the table on the way out with both operands in 4-bit floating point, a power of two for each block of 32

The plain forms below define the arithmetic.
"""
import math

import torch

own = False

VOCAB = 33708           # shared sub-word vocabulary of the tied weight
E4M3_MAX, E2M1_MAX = 448.0, 6.0
EPS = 1e-6
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # one answer being generated: the drawn token's log probability and 20 alternatives
        {"name": "logprob one row", "op": "logprob", "mode": "score", "rows": 1, "vocab": VOCAB, "x": "f32", "out": "f32", "top": 20, "masked": False, "scale": 1.0},
        # a large batch of requests under a grammar that forbids part of the vocabulary
        {"name": "logprob batch", "op": "logprob", "mode": "score", "rows": 512, "vocab": 65536, "x": "bf16", "out": "bf16", "top": 5, "masked": True, "scale": 1.0},
        # a base-size training step's loss and the gradient that the projection's backward takes
        {"name": "logprob loss base", "op": "logprob", "mode": "loss", "rows": 4096, "vocab": VOCAB, "x": "bf16", "out": "bf16", "top": 0, "masked": False, "scale": 1.0},
        # a big-size policy update with an entropy term at a temperature, tokens that fill no tile
        {"name": "logprob policy big", "op": "logprob", "mode": "policy", "rows": 8111, "vocab": VOCAB, "x": "f32", "out": "f32", "top": 0, "masked": False, "scale": 1.25},
        # a sub-layer of a base-size step, both ways
        {"name": "norm base", "op": "norm", "mode": "train", "rows": 8192, "d": 512, "x": "bf16", "residual": True, "pad": 0},
        # odd rows, not aligned, in a wider buffer
        {"name": "norm odd", "op": "norm", "mode": "train", "rows": 12801, "d": 1021, "x": "f32", "residual": True, "pad": 3},
        # a small batch's tokens being generated: the last norm and the logits
        {"name": "norm project", "op": "norm", "mode": "project", "rows": 48, "d": 1024, "vocab": VOCAB, "x": "bf16", "residual": True, "pad": 0},
        # the smallest training case of this repository: latency
        {"name": "clip tiny", "op": "clip", "vocab": 1000, "d": 64, "layers": 2, "layer": "f32", "clips": True},
        # all gradients of a big-size step, the layers' ones in 16 bits
        {"name": "clip big", "op": "clip", "vocab": VOCAB, "d": 1024, "layers": 12, "layer": "bf16", "clips": True},
        # one token being generated
        {"name": "project4 one token", "op": "project4", "update": False, "tokens": 1, "d": 1024, "vocab": VOCAB, "x": "bf16", "out": "f32"},
        # a beam search's or a small batch's tokens being generated
        {"name": "project4 batch", "op": "project4", "update": False, "tokens": 48, "d": 512, "vocab": VOCAB, "x": "bf16", "out": "bf16"},
        # a validation batch scored with a weight that has just changed
        {"name": "project4 scoring", "op": "project4", "update": True, "tokens": 4096, "d": 1024, "vocab": VOCAB, "x": "bf16", "out": "bf16"},
    ]


def _between(rng, low, high):
    """A whole number, spread evenly over the logarithm."""
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 1)))))))


def draw(rng):
    op = rng.choice(["logprob", "norm", "clip", "project4"])
    if op == "logprob":
        mode, x = rng.choice(["score", "loss", "policy"]), rng.choice(["f32", "bf16"])
        return {"op": op, "mode": mode, "rows": _between(rng, 1, 512 if mode == "score" else 4096), "vocab": rng.choice([1000, VOCAB, 65536, rng.randint(500, 65536)]), "x": x,
                "out": x if rng.random() < 0.7 else rng.choice(["f32", "bf16"]), "top": rng.choice([0, 1, 5, 20]) if mode == "score" else 0, "masked": rng.choice([True, False]),
                "scale": rng.choice([1.0, 1.25, 0.5])}
    if op == "norm":
        mode = rng.choice(["train", "train", "project"])
        case = {"op": op, "mode": mode, "rows": _between(rng, 1, 12800 if mode == "train" else 512), "d": rng.choice([64, 512, 1024, 8 * rng.randint(8, 128), rng.randint(33, 1024)]),
                "x": rng.choice(["f32", "bf16"]), "residual": rng.choice([True, True, False]), "pad": rng.choice([0, 0, 8, rng.randint(1, 63)])}
        if mode == "project":
            case["vocab"] = rng.choice([1000, VOCAB, rng.randint(1000, VOCAB)])
        return case
    if op == "clip":
        return {"op": op, "vocab": rng.choice([1000, VOCAB]), "d": rng.choice([64, 512, rng.randint(33, 700)]), "layers": rng.randint(0, 12), "layer": rng.choice(["f32", "bf16"]), "clips": rng.choice([True, True, False])}
    return {"op": op, "update": rng.choice([True, False]), "tokens": _between(rng, 1, 4000), "d": rng.choice([512, 1024, rng.randint(64, 1024)]), "vocab": rng.choice([1000, VOCAB, rng.randint(1000, VOCAB)]),
            "x": rng.choice(["f32", "bf16"]), "out": rng.choice(["f32", "bf16"])}


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
    s = {"case": case}
    op = case["op"]
    if op == "logprob":
        n, vocab = case["rows"], case["vocab"]
        unigram = -1.1 * torch.log(torch.arange(1, vocab + 1, device="cuda", dtype=torch.float32))
        logits = torch.randn(n, vocab, device="cuda", generator=g).mul_(2).add_(unigram + 12)
        targets = _zipf(n, vocab, g)
        if case["masked"]:  # three in ten tokens cannot follow; the given one can
            at = torch.arange(n, device="cuda")
            kept = logits[at, targets]
            logits.masked_fill_(torch.rand(n, vocab, device="cuda", generator=g) < 0.3, -math.inf)
            logits[at, targets] = kept
        s["logits"] = logits.to(TYPES[case["x"]])
        padding = torch.rand(n, device="cuda", generator=g) < (0.0 if case["mode"] == "score" else 0.1)
        s["targets"] = targets.masked_fill(padding, -1)  # rows of padding have no token
        s["dlogprob"] = torch.full((n,), -1.0 / n, device="cuda") if case["mode"] == "loss" else torch.randn(n, device="cuda", generator=g) / n
        s["dentropy"] = (0.01 / n) * (1 + torch.rand(n, device="cuda", generator=g)) * ~padding
        new = lambda *shape: torch.empty(*shape, device="cuda")  # noqa: E731
        s["logprob"], s["stats"], s["entropy"] = new(n), new(n, 2), new(n)
        if case["top"]:
            s["top_tokens"], s["top_logprob"] = torch.empty(n, case["top"], device="cuda", dtype=torch.int64), new(n, case["top"])
        if case["mode"] != "score":
            s["dlogits"] = torch.empty(n, vocab, device="cuda", dtype=TYPES[case["out"]])
    elif op == "norm":
        n, d, pad, dtype = case["rows"], case["d"], case["pad"], TYPES[case["x"]]
        s["x"] = _padded(n, d, pad, dtype, g)
        s["residual"] = (_padded(n, d, pad, dtype, g).float() * 3).to(dtype) if case["residual"] else None
        s["weight"] = 1 + 0.2 * torch.randn(d, device="cuda", generator=g)
        s["sum"] = torch.empty(n, d, device="cuda", dtype=dtype) if case["residual"] else None
        if case["mode"] == "train":
            s["grad"], s["dsum"] = _padded(n, d, pad, dtype, g), _padded(n, d, pad, dtype, g)
            s["out"], s["dx"] = (torch.empty(n, d, device="cuda", dtype=dtype) for _ in range(2))
            s["inv_rms"], s["dweight"] = torch.empty(n, device="cuda"), torch.empty(d, device="cuda")
        else:
            vocab = case["vocab"]
            s["table"] = torch.randn(vocab, d, device="cuda", generator=g) * d ** -0.5
            s["q"], s["q_scale"] = _square(s["table"])  # kept between calls
            s["logits"] = torch.empty(n, vocab, device="cuda", dtype=torch.bfloat16)
        if own:
            import paper_1905_04035_b200 as dst
            if case["mode"] == "train":
                s["workspace"] = torch.empty(dst.dst_rmsnorm_backward_workspace_bytes(n, d), device="cuda", dtype=torch.uint8)
            else:
                s["rows8"] = dst.Fp8Matrix(n, d)
                s["projection"] = dst.TiedProjection(vocab, d, n, training=False)
                s["projection"].update(s["table"])
    elif op == "clip":
        vocab, d, layers, layer = case["vocab"], case["d"], case["layers"], TYPES[case["layer"]]
        shapes = [((vocab, d), torch.float32)] + [(shape, layer) for _ in range(layers) for shape in ((4 * d, d), (8 * d, d), (4 * d,), (d,))]
        s["grads"] = [(torch.randn(shape, device="cuda", generator=g) * 1e-3).to(dtype) for shape, dtype in shapes]
        s["outs"] = [torch.empty_like(t) for t in s["grads"]]
        size = sum(t.numel() for t in s["grads"])
        s["max_norm"] = 1e-3 * size ** 0.5 * (0.3 if case["clips"] else 3.0)
        s["clip"] = torch.empty(2, device="cuda")
        if own:
            import paper_1905_04035_b200 as dst
            s["list"], s["out_list"] = dst.TensorList(s["grads"]), dst.TensorList(s["outs"])
            s["workspace"] = torch.empty(dst.dst_grad_norm_workspace_bytes(s["list"]), device="cuda", dtype=torch.uint8)
    else:
        m, d, vocab = case["tokens"], case["d"], case["vocab"]
        s["x"] = torch.randn(m, d, device="cuda", generator=g).to(TYPES[case["x"]])
        s["weight"] = torch.randn(vocab, d, device="cuda", generator=g) * d ** -0.5
        s["logits"] = torch.empty(m, vocab, device="cuda", dtype=TYPES[case["out"]])
        if not case["update"]:  # the weight stays as it is between calls: its 4-bit form is kept
            s["codes"], s["unit"] = _codes4(s["weight"])
        if own:
            import paper_1905_04035_b200 as dst
            s["projection"] = dst.TiedProjection(vocab, d, m, training=False, bits=4)
            if not case["update"]:
                s["projection"].update(s["weight"])
    return s


# ---- plain forms -------------------------------------------------------------------------------------------------
def _power(amax, most):
    """The smallest power of two 2^e with amax <= most * 2^e."""
    mantissa, exponent = torch.frexp(amax.clamp_min(2.0 ** -100))
    top, top_exponent = math.frexp(most)
    return torch.ldexp(torch.ones_like(amax), exponent - top_exponent + (mantissa > top).int())


def _blocks(x, size):
    return torch.nn.functional.pad(x.float(), (0, -x.shape[1] % size)).view(x.shape[0], -1, size)


def _rounded8(x):
    """x as its 8-bit form stands for it: one scale for every 128 consecutive elements of a row."""
    b = _blocks(x, 128)
    scale = _power(b.abs().amax(-1, keepdim=True), E4M3_MAX)
    return ((b / scale).to(torch.float8_e4m3fn).float() * scale).reshape(x.shape[0], -1)[:, :x.shape[1]]


def _square(w):
    """8-bit form of w with one scale for every 128 x 128 block."""
    rows, cols = w.shape
    b = torch.nn.functional.pad(w.float(), (0, -cols % 128, 0, -rows % 128))
    b = b.view(b.shape[0] // 128, 128, -1, 128)
    scale = _power(b.abs().amax((1, 3), keepdim=True), E4M3_MAX)
    return (b / scale).to(torch.float8_e4m3fn), scale


def _of_square(q, scale, shape):
    b = q.float() * scale
    return b.reshape(b.shape[0] * 128, -1)[:shape[0], :shape[1]]


def _codes4(x):
    """x in 4 bits (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives) and the scale of every 32 consecutive elements of a row."""
    b = _blocks(x, 32)
    scale = _power(b.abs().amax(-1, keepdim=True), E2M1_MAX)
    v = b / scale
    a = v.abs()
    step = 0.5 + 0.5 * (a >= 2) + (a >= 4)
    return torch.round(v / step) * step, scale


def _of_codes4(codes, scale, cols):
    return (codes * scale).reshape(codes.shape[0], -1)[:, :cols]


def _logprob(s):
    c = s["case"]
    x = s["logits"].float()
    z = (x - x.amax(-1, keepdim=True)) * c["scale"]
    e = torch.exp(z)
    total = e.sum(-1, keepdim=True)
    z = z.clamp_min(-1e4)  # a weight of zero times its logarithm is zero
    log_total = torch.log(total)
    entropy = log_total - (e * z).sum(-1, keepdim=True) / total
    at = s["targets"].clamp_min(0).view(-1, 1)
    given = s["targets"].view(-1, 1) >= 0
    r = {"logprob": torch.where(given, z.gather(-1, at) - log_total, 0.0).view(-1), "entropy": entropy.view(-1)}
    if c["top"]:
        order = torch.sort(x, dim=-1, descending=True, stable=True)[1][:, :c["top"]]
        r |= {"top_tokens": order, "top_logprob": z.gather(-1, order) - log_total}
    if c["mode"] != "score":
        p = e / total
        weight = torch.where(given, s["dlogprob"].view(-1, 1), 0.0)
        grad = -p * weight if c["mode"] == "loss" else -p * (weight + s["dentropy"].view(-1, 1) * (z - log_total + entropy))
        grad.scatter_add_(-1, at, weight)
        r["dlogits"] = (grad * c["scale"]).to(s["dlogits"].dtype)
    return r


def _norm(s):
    c = s["case"]
    dtype, w = s["x"].dtype, s["weight"]
    h = s["x"].float()
    if s["residual"] is not None:
        h = (h + s["residual"].float()).to(dtype)
        r = {"sum": h}
        h = h.float()
    else:
        r = {}
    inv = torch.rsqrt(h.square().mean(-1, keepdim=True) + EPS)
    y = h * inv * w
    if c["mode"] == "project":
        table = _of_square(s["q"], s["q_scale"], (c["vocab"], c["d"]))
        return r | {"logits": (_rounded8(y) @ table.T).to(torch.bfloat16)}
    unit, dy = h * inv, s["grad"].float()
    g = dy * w
    dx = s["dsum"].float() + inv * (g - unit * (g * unit).mean(-1, keepdim=True))
    return r | {"out": y.to(dtype), "dx": dx.to(dtype), "dweight": (dy * unit).sum(0)}


def run(s):
    c, op = s["case"], s["case"]["op"]
    if own:
        import paper_1905_04035_b200 as dst
        if op == "logprob":
            x, t, scale = s["logits"], s["targets"], c["scale"]
            r = {"logprob": s["logprob"], "entropy": s["entropy"]}
            if c["mode"] == "score":
                top = {"top_tokens": s["top_tokens"], "top_logprob": s["top_logprob"]} if c["top"] else {}
                dst.dst_logprob(x, t, s["logprob"], scale=scale, entropy=s["entropy"], **top)
                return r | top
            if c["mode"] == "loss":
                dst.dst_logprob_loss(x, t, s["dlogprob"], s["logprob"], s["dlogits"], scale=scale, entropy=s["entropy"])
            else:
                dst.dst_logprob(x, t, s["logprob"], scale=scale, stats=s["stats"], entropy=s["entropy"])
                dst.dst_logprob_backward(x, t, s["stats"], s["dlogprob"], s["dlogits"], scale=scale, entropy=s["entropy"], dentropy=s["dentropy"])
            return r | {"dlogits": s["dlogits"]}
        if op == "norm":
            added = {} if s["residual"] is None else {"residual": s["residual"], "sum_out": s["sum"]}
            r = {} if s["residual"] is None else {"sum": s["sum"]}
            if c["mode"] == "project":
                dst.dst_rmsnorm(s["x"], s["weight"], q=s["rows8"], eps=EPS, **added)
                return r | {"logits": s["projection"].logits(s["rows8"], s["logits"])}
            dst.dst_rmsnorm(s["x"], s["weight"], s["out"], eps=EPS, inv_rms=s["inv_rms"], **added)
            h = s["x"] if s["residual"] is None else s["sum"]
            dst.dst_rmsnorm_backward(s["grad"], h, s["weight"], s["inv_rms"], s["dx"], dsum=s["dsum"], dweight=s["dweight"], workspace=s["workspace"])
            return r | {"out": s["out"], "dx": s["dx"], "dweight": s["dweight"]}
        if op == "clip":
            dst.dst_grad_norm(s["list"], s["clip"], s["max_norm"], s["workspace"])
            dst.dst_clip(s["list"], s["clip"], s["out_list"])
            return {"norm": s["clip"], "grads": s["outs"]}
        if c["update"]:
            s["projection"].update(s["weight"])
        return {"logits": s["projection"].logits(s["x"], s["logits"])}
    if op == "logprob":
        return _logprob(s)
    if op == "norm":
        return _norm(s)
    if op == "clip":
        squares = torch.stack([t.float().square().sum() for t in s["grads"]])
        norm = squares.sum().sqrt()
        factor = (s["max_norm"] / (norm + 1e-6)).clamp_max(1.0)
        return {"norm": torch.stack([norm, factor]), "grads": [(t.float() * factor).to(t.dtype) for t in s["grads"]]}
    codes, unit = _codes4(s["weight"]) if c["update"] else (s["codes"], s["unit"])
    return {"logits": (_of_codes4(*_codes4(s["x"]), c["d"]) @ _of_codes4(codes, unit, c["d"]).T).to(s["logits"].dtype)}


# ---- what a pass cannot do without -------------------------------------------------------------------------------
def work(case):
    size = lambda t: 4 if t == "f32" else 2  # noqa: E731
    op = case["op"]
    if op == "logprob":
        n, entries = case["rows"], case["rows"] * case["vocab"]
        if case["mode"] == "score":
            return {"bytes": entries * size(case["x"]) + n * (16 + 12 * case["top"]), "flops": 6 * entries}
        return {"bytes": entries * (size(case["x"]) + size(case["out"])) + n * 24, "flops": 12 * entries}
    if op == "norm":
        n, d, x, more = case["rows"], case["d"], size(case["x"]), 2 * bool(case["residual"])
        if case["mode"] == "project":
            return {"bytes": n * d * x * (1 + more) + case["vocab"] * d + n * case["vocab"] * 2, "flops": 2 * n * d * case["vocab"]}
        return {"bytes": n * d * x * (5 + more) + 8 * d, "flops": 16 * n * d}
    if op == "clip":
        table, layers = case["vocab"] * case["d"], case["layers"] * (12 * case["d"] ** 2 + 5 * case["d"])
        return {"bytes": 2 * (table * 4 + layers * size(case["layer"])), "flops": 3 * (table + layers)}
    m, d, vocab = case["tokens"], case["d"], case["vocab"]
    return {"bytes": m * d * size(case["x"]) + (vocab * d * 4 if case["update"] else vocab * (d // 2 + -(-d // 32))) + m * vocab * size(case["out"]), "flops": 2 * m * d * vocab}


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------
def _exact_rounded(x, rows, cols, most, bits, least):
    """x in 64 bits with `bits` bits after the leading one, `least` the smallest exponent of the type, and one power of two for each block of rows x cols."""
    x = x.double()
    n, m = x.shape
    full = x.new_zeros(-(-n // rows) * rows, -(-m // cols) * cols)
    full[:n, :m] = x
    b = full.unfold(0, rows, rows).unfold(1, cols, cols)
    unit = torch.exp2(torch.ceil(torch.log2(b.abs().amax((2, 3)).clamp_min(2.0 ** -100) / most)))
    unit = unit.repeat_interleave(rows, 0).repeat_interleave(cols, 1)[:n, :m]
    v = x / unit
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp_min(2.0 ** least))) - bits)
    return torch.round(v / step) * step * unit


def _exact_logprob(s):
    c = s["case"]
    x = s["logits"].double() * c["scale"]
    lse = torch.logsumexp(x, -1)
    log_p = x.sub_(lse.view(-1, 1))
    p = torch.exp(log_p)
    log_p = torch.where(p > 0, log_p, 0.0)
    entropy = -(p * log_p).sum(-1)
    rows = torch.arange(c["rows"], device="cuda")
    given = s["targets"] >= 0
    token = torch.where(given, s["targets"], 0)
    r = {"logprob": torch.where(given, log_p[rows, token], 0.0), "entropy": entropy}
    if c["top"]:
        # the tokens are whole numbers: by the logit, then by the index
        key = s["logits"].double().cpu().numpy()
        import numpy as np
        order = torch.from_numpy(np.stack([np.lexsort((np.arange(len(k)), -k))[:c["top"]] for k in key])).cuda()
        r |= {"top_tokens": order, "top_logprob": log_p.gather(-1, order)}
    if c["mode"] != "score":
        weight = s["dlogprob"].double() * given
        grad = p * -weight.view(-1, 1)
        if c["mode"] == "policy":
            grad -= p * (log_p + entropy.view(-1, 1)) * s["dentropy"].double().view(-1, 1)
        grad[rows, token] += weight
        r["dlogits"] = grad * c["scale"]
    return r


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "logprob":
        return _exact_logprob(s)
    if op == "norm":
        h = s["x"].double()
        r = {}
        if s["residual"] is not None:
            r["sum"] = h + s["residual"].double()
            h = r["sum"].to(s["x"].dtype).double()  # the norm is that of the stream as it is stored
        inv = (h.pow(2).sum(-1, keepdim=True) / case["d"] + EPS) ** -0.5
        unit, w = h * inv, s["weight"].double()
        if case["mode"] == "project":
            table = _exact_rounded(s["table"], 128, 128, E4M3_MAX, 3, -6)
            return r | {"logits": torch.mm(_exact_rounded(unit * w, 1, 128, E4M3_MAX, 3, -6), table.T)}
        dy = s["grad"].double()
        along = torch.einsum("nd,nd->n", dy * w, unit) / case["d"]
        return r | {"out": unit * w, "dx": s["dsum"].double() + (dy * w - unit * along.view(-1, 1)) * inv, "dweight": torch.einsum("nd,nd->d", dy, unit)}
    if op == "clip":
        norm = math.sqrt(math.fsum(float(torch.linalg.vector_norm(t.double())) ** 2 for t in s["grads"]))
        factor = min(1.0, s["max_norm"] / (norm + 1e-6))
        return {"norm": torch.tensor([norm, factor], dtype=torch.float64), "grads": [t.double() * factor for t in s["grads"]]}
    return {"logits": torch.mm(_exact_rounded(s["x"], 1, 32, E2M1_MAX, 1, 0), _exact_rounded(s["weight"], 1, 32, E2M1_MAX, 1, 0).T)}
