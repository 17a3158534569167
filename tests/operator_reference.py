"""The training operators written from their formulas in 64 bits (torch, any device)."""
import torch

COEFS = (3.4445, -4.7750, 2.0315)


def orthogonalize(G, steps=5, coefs=COEFS, eps=1e-7):
    a, b, c = coefs
    x = G.double()
    x = x / (x.square().sum((-2, -1), keepdim=True).sqrt() + eps)
    for _ in range(steps):
        A = x @ x.mT if x.shape[-2] <= x.shape[-1] else x.mT @ x
        P = b * A + c * (A @ A)
        x = a * x + (P @ x if x.shape[-2] <= x.shape[-1] else x @ P)
    return x


def muon(W, V, G, lr, mu, nesterov, weight_decay, scale, **kw):
    v = mu * V.double() + G.double()
    u = G.double() + mu * v if nesterov else v
    return (1 - lr * weight_decay) * W.double() - lr * scale * orthogonalize(u, **kw), v


def alive(logits, live):
    on = torch.ones(logits.shape[:2], dtype=torch.bool, device=logits.device) if live is None else live != 0
    return on & ~(logits == float("-inf")).all(-1)


def choose(logits, k, on):
    """The k largest logits of every live token, ties to the lowest index; -1 elsewhere."""
    order = torch.sort(logits.double(), dim=-1, descending=True, stable=True).indices[..., :k]
    return torch.where(on[..., None], order, -1)


def route(logits, k, coef, normalize=False, live=None):
    G, T, E = logits.shape
    on = alive(logits, live)
    chosen = choose(logits, k, on)
    p = torch.softmax(torch.where(on[..., None], logits.double(), 0.0), -1) * on[..., None]
    w = p.gather(-1, chosen.clamp(min=0)) * on[..., None]
    if normalize:
        w = torch.where(on[..., None], w / w.sum(-1, keepdim=True), 0.0)
    counts = torch.stack([torch.bincount(chosen[g][on[g]].reshape(-1), minlength=E) for g in range(G)]) if T else torch.zeros(G, E, dtype=torch.long, device=logits.device)
    n = on.sum(1, keepdim=True).clamp(min=1).double()
    mean = p.sum(1) / n
    loss = coef * E * (counts / (k * n) * mean).sum(1)
    return chosen, w, counts, mean, loss


def route_objective(x, chosen, counts, on, coef, normalize, dweights, dloss):
    """sum dloss loss + sum dweights weights as a function of the logits x (64 bits), choice and counts held fixed."""
    E, k = x.shape[-1], chosen.shape[-1]
    p = torch.softmax(torch.where(on[..., None], x, 0.0), -1) * on[..., None]
    n = (counts.sum(1, keepdim=True).double() / k).clamp(min=1)
    total = x.new_zeros(())
    if dloss is not None:
        total = total + (dloss.double() * coef * E * (counts.double() / (k * n) * (p.sum(1) / n)).sum(1)).sum()
    if dweights is not None:
        w = p.gather(-1, chosen.long().clamp(min=0))
        if normalize:
            w = w / torch.where(on[..., None], w.sum(-1, keepdim=True), 1.0)
        total = total + (w * on[..., None] * dweights.double()).sum()
    return total


def route_grad(logits, chosen, counts, coef, normalize=False, live=None, dweights=None, dloss=None):
    on = alive(logits, live)
    x = torch.where(on[..., None], logits.double(), 0.0).requires_grad_(True)
    f = route_objective(x, chosen, counts, on, coef, normalize, dweights, dloss)
    return torch.autograd.grad(f, x)[0] if f.requires_grad else torch.zeros_like(x)
