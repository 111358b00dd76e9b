"""A language model of one residual layer around one tied weight, trained and then sampled from: every use of the weight
runs through the library.

    rows in     dst_embed                (lookup, scale, positions, dropout)
    layer       torch.matmul, then dst_dropout onto the residual stream
    logits      TiedProjection.logits    (8-bit product; the loss is torch's)
    gradients   TiedProjection.backward  (dx, and dweight = the dense partner)
                dst_dropout              (of the layer, and of the embedding: the value rows)
    step        dst_densify_apply        (value rows + dense partner -> Adam on the fp32 weight)
    answers     TiedProjection.logits, dst_sample

The task is synthetic: the next token is a fixed permutation of the present one, with Zipf-distributed tokens.
Run: python -m examples.tied_training [--steps N]
"""
import argparse

import torch

import paper_1905_04035_b200 as dst


class TiedModel:
    def __init__(self, vocab=1000, d=128, tokens=512, p=0.1, seed=0, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        self.vocab, self.d, self.tokens, self.p, self.seed, self.scale = vocab, d, tokens, p, seed, d ** 0.5
        self.weight = torch.randn(vocab, d, device=device, generator=g) * d ** -0.5
        self.layer = torch.randn(d, d, device=device, generator=g) * 0.02
        self.position = torch.zeros(tokens, d, device=device)
        self.state1, self.state2 = torch.zeros_like(self.weight), torch.zeros_like(self.weight)
        self.projection = dst.TiedProjection(vocab, d, tokens, device=device)
        self.projection.update(self.weight)
        new = lambda *shape: torch.empty(*shape, device=device)  # noqa: E731
        self.x, self.h, self.dh, self.du, self.values = (new(tokens, d) for _ in range(5))
        self.logits, self.dweight = new(tokens, vocab), new(vocab, d)
        self.workspace = torch.empty(dst.dst_workspace_bytes(tokens, 1, d, vocab), dtype=torch.uint8, device=device)

    def forward(self, tokens, step, p):
        """Logits of a batch of tokens; dropout's bits follow from the step alone."""
        n = tokens.shape[0]
        x, h = self.x[:n], self.h[:n]
        dst.dst_embed(tokens, self.weight, x, scale=self.scale, position=self.position, p=p, seed=self.seed, offset=2 * step)
        dst.dst_dropout(x @ self.layer, h, p, self.seed, 2 * step + 1, residual=x)
        return self.projection.logits(h, self.logits[:n])

    def train_step(self, tokens, targets, step, lr=2e-3):
        logits = self.forward(tokens, step, self.p)
        n = tokens.shape[0]
        log_prob = torch.log_softmax(logits, -1)
        rows = torch.arange(n, device=logits.device)
        loss = -log_prob[rows, targets].mean()
        dlogits = log_prob.exp()
        dlogits[rows, targets] -= 1
        dlogits /= n
        self.projection.backward(dlogits, self.h, self.dh, self.dweight)
        dst.dst_dropout(self.dh, self.du, self.p, self.seed, 2 * step + 1)        # through the layer's dropout
        dx = self.dh + self.du @ self.layer.T
        self.layer -= 0.1 * (self.x.T @ self.du)
        dst.dst_dropout(dx, self.values, self.p, self.seed, 2 * step, scale=self.scale)
        dst.dst_densify_apply([(tokens, self.values)], self.d, self.vocab, self.dweight, self.weight, self.workspace,
                              kind=dst.DST_OPT_ADAM, lr=lr, step=step + 1, state1=self.state1, state2=self.state2)
        self.projection.update(self.weight)
        return loss

    def answer(self, tokens, uniform, **filters):
        """The next token of each given one, drawn with the given uniform numbers."""
        out = torch.empty(tokens.shape[0], dtype=torch.int64, device=tokens.device)
        return dst.dst_sample(self.forward(tokens, 0, 0.0), uniform, out, **filters)


def train(steps=200, seed=0):
    """(losses, share of right answers)."""
    model = TiedModel(seed=seed)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    follows = torch.randperm(model.vocab, device="cuda", generator=g)
    weights = torch.arange(1, model.vocab + 1, device="cuda", dtype=torch.float32) ** -1.1
    batch = lambda n: torch.multinomial(weights, n, replacement=True, generator=g)  # noqa: E731
    losses = []
    for step in range(steps):
        tokens = batch(model.tokens)
        losses.append(model.train_step(tokens, follows[tokens], step))
    tokens = batch(256)
    n = tokens.shape[0]
    full = lambda v, dtype=torch.float32: torch.full((n,), v, dtype=dtype, device="cuda")  # noqa: E731
    drawn = model.answer(tokens, torch.rand(n, device="cuda", generator=g), temperature=full(0.7), top_k=full(40, torch.int32), top_p=full(0.95), min_p=full(0.02))
    return [float(v) for v in losses], float((drawn == follows[tokens]).float().mean())


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=200)
    steps = ap.parse_args().steps
    losses, right = train(steps)
    for i in range(0, steps, max(1, steps // 10)):
        print("step %4d  loss %.3f" % (i, losses[i]))
    print("last loss %.3f; %.0f %% of the sampled next tokens are right" % (losses[-1], 100 * right))
