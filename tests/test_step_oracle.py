"""The definitions in oracle/step_oracle.py against hand-worked numbers, torch in 64 bits, and differences."""
import numpy as np
import torch

from oracle import step_oracle as o


def test_log_probabilities_by_hand_and_by_torch():
    log_p, lse, entropy, r = o.log_probabilities([[0.0, np.log(3.0)]])
    assert np.allclose(np.exp(log_p), [[0.25, 0.75]]) and np.isclose(lse[0], np.log(4)) and np.isclose(r[0], 1 / 3)
    assert np.isclose(entropy[0], -(0.25 * np.log(0.25) + 0.75 * np.log(0.75)))
    x = np.random.default_rng(0).normal(size=(5, 40)) * 3
    x[1, ::2] = -np.inf
    log_p, lse, entropy, _ = o.log_probabilities(x, 1.5)
    t = torch.log_softmax(torch.from_numpy(x) * 1.5, -1)
    assert np.allclose(log_p, t.numpy()) and np.allclose(lse, torch.logsumexp(torch.from_numpy(x) * 1.5, -1).numpy())
    p = t.exp()
    assert np.allclose(entropy, -(torch.where(p > 0, p * t, 0.0)).sum(-1).numpy())
    log_p, lse, entropy, r = o.log_probabilities([[-np.inf, -np.inf], [0.0, -50.0]])
    assert np.all(log_p[0] == -np.inf) and lse[0] == -np.inf and entropy[0] == 0 and r[0] == -1
    assert np.isclose(log_p[1, 0], -np.exp(-50.0), rtol=1e-12)      # relative to itself, not to one


def test_special_values_of_log_probabilities():
    log_p, lse, entropy, _ = o.log_probabilities([[0.0, np.nan], [0.0, np.inf]])
    assert np.isnan(log_p[0]).all() and np.isnan(lse).all() and np.isnan(entropy).all()


def test_top_tokens():
    x = [[1.0, 3.0, 3.0, -np.inf, np.nan], [-np.inf] * 5]
    assert o.top_tokens(x, 4).tolist() == [[1, 2, 0, -1], [-1] * 4]


def test_logits_gradient_by_torch():
    g = np.random.default_rng(1)
    x, targets, a, b = g.normal(size=(4, 9)), np.array([3, -1, 0, 8]), g.normal(size=4), g.normal(size=4)
    t = torch.from_numpy(x).requires_grad_()
    log_p = torch.log_softmax(t * 0.7, -1)
    entropy = -(log_p.exp() * log_p).sum(-1)
    picked = log_p[torch.arange(4), torch.from_numpy(targets).clamp_min(0)] * torch.from_numpy(targets >= 0)
    (picked * torch.from_numpy(a) + entropy * torch.from_numpy(b)).sum().backward()
    assert np.allclose(o.logits_gradient(x, targets, 0.7, a, b), t.grad.numpy())
    assert np.all(o.logits_gradient(x, targets, 0.7, a * 0, b * 0) == 0)


def test_rmsnorm_by_torch():
    g = np.random.default_rng(2)
    h, w, dy, ds = g.normal(size=(3, 8)), g.normal(size=8), g.normal(size=(3, 8)), g.normal(size=(3, 8))
    th, tw = torch.from_numpy(h).requires_grad_(), torch.from_numpy(w).requires_grad_()
    y = th * torch.rsqrt((th * th).mean(-1, keepdim=True) + 1e-3) * tw
    (y * torch.from_numpy(dy)).sum().backward()
    want, inv = o.rmsnorm(h, w, 1e-3)
    dx, dw = o.rmsnorm_gradient(dy, h, w, inv, ds)
    assert np.allclose(want, y.detach().numpy()) and np.allclose(dx, th.grad.numpy() + ds) and np.allclose(dw, tw.grad.numpy())


def test_clip():
    norm, factor, out = o.clip([np.array([3.0]), np.array([[4.0]])], 1.0)
    assert norm == 5.0 and np.isclose(factor, 0.2, rtol=1e-6) and np.isclose(out[1][0, 0], 0.8, rtol=1e-6)
    assert o.clip([np.array([3.0])], 10.0)[1] == 1.0
    assert o.clip([np.array([np.inf, 1.0])], 1.0)[1:][0] == 0.0 and np.all(o.clip([np.array([np.nan])], 1.0)[2][0] == 0)
