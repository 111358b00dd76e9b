"""The model of tied_training with a norm before the projection, its loss and clipping through the library too, answers in 4 bits
with their log probabilities:

    residual   dst_dropout of the layer's output, then dst_rmsnorm: the stream's sum, its norm, and the norm in 8 bits
    logits     TiedProjection.logits of the 8-bit rows
    loss       dst_logprob_loss           (log probabilities, and the logits' gradient in their place)
    gradients  TiedProjection.backward, dst_rmsnorm_backward, dst_dropout
    table      dst_densify                (value rows + dense partner -> one gradient)
    clipping   dst_grad_norm, dst_clip    (over the table's, the layer's and the norm's gradients)
    step       dst_densify_apply          (Adam on the table; the small weights take plain steps)
    answers    TiedProjection(bits=4).logits, dst_sample, dst_logprob with alternatives

Run: python -m examples.tied_step [--steps N]
"""
import argparse

import torch

import paper_1905_04035_b200 as dst

from .tied_training import TiedModel


class NormedModel(TiedModel):
    def __init__(self, vocab=1000, d=128, tokens=512, p=0.1, seed=0, max_norm=1.0, device="cuda"):
        super().__init__(vocab, d, tokens, p, seed, device)
        new = lambda *shape: torch.empty(*shape, device=device)  # noqa: E731
        self.max_norm = max_norm
        self.gain, self.dgain = torch.ones(d, device=device), new(d)
        self.y, self.dy, self.inv_rms, self.logprob = new(tokens, d), new(tokens, d), new(tokens), new(tokens)
        self.rows8 = dst.Fp8Matrix(tokens, d, device=device)
        self.dlayer = new(d, d)
        self.norm_workspace = torch.empty(dst.dst_rmsnorm_backward_workspace_bytes(tokens, d), dtype=torch.uint8, device=device)
        self.grads = dst.TensorList([self.dweight, self.dlayer, self.dgain])
        self.clip = new(2)
        self.clip_workspace = torch.empty(dst.dst_grad_norm_workspace_bytes(self.grads), dtype=torch.uint8, device=device)
        self.answers = dst.TiedProjection(vocab, d, tokens, training=False, bits=4, device=device)

    def stream(self, tokens, step, p):
        """The rows before the projection, normed, in 32 and in 8 bits; the residual stream stays in ``h``."""
        n = tokens.shape[0]
        x, h, y, rows8 = self.x[:n], self.h[:n], self.y[:n], self.rows8.part(n, self.d)
        dst.dst_embed(tokens, self.weight, x, scale=self.scale, position=self.position, p=p, seed=self.seed, offset=2 * step)
        u = x @ self.layer
        dst.dst_dropout(u, u, p, self.seed, 2 * step + 1)
        dst.dst_rmsnorm(u, self.gain, y, q=rows8, residual=x, sum_out=h, inv_rms=self.inv_rms[:n])
        return y, rows8

    def gradients(self, tokens, targets, step):
        """The loss; gradients of the table, the layer and the norm in dweight, dlayer and dgain.  Targets below zero are padding."""
        n = tokens.shape[0]
        y, rows8 = self.stream(tokens, step, self.p)
        logits, logprob = self.projection.logits(rows8, self.logits[:n]), self.logprob[:n]
        weight = -(targets >= 0).float()
        weight /= -weight.sum()
        dst.dst_logprob_loss(logits, targets, weight, logprob, logits)
        dy, dh, du, values, inv_rms = self.dy[:n], self.dh[:n], self.du[:n], self.values[:n], self.inv_rms[:n]
        self.projection.backward(logits, y, dy, self.dweight)
        dst.dst_rmsnorm_backward(dy, self.h[:n], self.gain, inv_rms, dh, dweight=self.dgain, workspace=self.norm_workspace)
        dst.dst_dropout(dh, du, self.p, self.seed, 2 * step + 1)                  # through the layer's dropout
        torch.mm(self.x[:n].T, du, out=self.dlayer)
        dst.dst_dropout(dh + du @ self.layer.T, values, self.p, self.seed, 2 * step, scale=self.scale)
        dst.dst_densify(tokens, values, self.d, self.vocab, self.dweight, self.dweight, self.workspace)
        return (logprob * weight).sum()

    def train_step(self, tokens, targets, step, lr=2e-3):
        loss = self.gradients(tokens, targets, step)
        dst.dst_grad_norm(self.grads, self.clip, self.max_norm, self.clip_workspace)
        dst.dst_clip(self.grads, self.clip)
        self.layer -= 0.1 * self.dlayer
        self.gain -= 0.1 * self.dgain
        dst.dst_densify_apply([], self.d, self.vocab, self.dweight, self.weight, self.workspace, kind=dst.DST_OPT_ADAM, lr=lr, step=step + 1,
                              state1=self.state1, state2=self.state2)
        self.projection.update(self.weight)
        return loss

    def answer(self, tokens, uniform, alternatives=3, **filters):
        """The next token of each given one, drawn with the given uniform numbers; its log probability and the likeliest tokens'."""
        n = tokens.shape[0]
        self.answers.update(self.weight)
        y, _ = self.stream(tokens, 0, 0.0)
        logits = self.answers.logits(y, self.logits[:n])
        drawn = torch.empty(n, dtype=torch.int64, device=tokens.device)
        dst.dst_sample(logits, uniform, drawn, **filters)
        logprob = torch.empty(n, device=tokens.device)
        others = torch.empty(n, alternatives, dtype=torch.int64, device=tokens.device)
        others_logprob = torch.empty(n, alternatives, device=tokens.device)
        dst.dst_logprob(logits, drawn, logprob, top_tokens=others, top_logprob=others_logprob)
        return drawn, logprob, others, others_logprob


def train(steps=200, seed=0):
    """(losses, share of right answers)."""
    model = NormedModel(seed=seed)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    follows = torch.randperm(model.vocab, device="cuda", generator=g)
    weights = torch.arange(1, model.vocab + 1, device="cuda", dtype=torch.float32) ** -1.1
    losses = []
    for step in range(steps):
        tokens = torch.multinomial(weights, model.tokens, replacement=True, generator=g)
        losses.append(model.train_step(tokens, follows[tokens], step))
    tokens = torch.multinomial(weights, 256, replacement=True, generator=g)
    drawn, _, _, _ = model.answer(tokens, torch.rand(256, device="cuda", generator=g), top_k=torch.full((256,), 40, dtype=torch.int32, device="cuda"))
    return [float(v) for v in losses], float((drawn == follows[tokens]).float().mean())


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=200)
    steps = ap.parse_args().steps
    losses, right = train(steps)
    for i in range(0, steps, max(1, steps // 10)):
        print("step %4d  loss %.3f" % (i, losses[i]))
    print("last loss %.3f; %.0f %% of the sampled next tokens are right" % (losses[-1], 100 * right))
