"""Cases of the training operators for stacked local workers: the Newton-Schulz orthogonalisation of a batch of
matrices, the Muon step built on it, the top-k router with its balance loss and per-expert counts, and the
router's gradient.  Every operator is written here in its plain form (elementary torch operations in fp32) and as
the call of the library that computes the same."""
import math

import torch

own = False

COEFS = (3.4445, -4.7750, 2.0315)
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
DEVICE = "cuda:0"


# ---- cases --------------------------------------------------------------------------------------------------
def listed():
    return [
        # the class layer 1024 -> 10 of 16 workers: the smallest call, where latency counts
        {"name": "ortho_16x10x1024_fp32", "op": "orthogonalize", "batch": 16, "rows": 10, "cols": 1024, "type": "fp32", "pad": 0},
        # odd sizes, taller than wide, rows of a wider array, fp32 results
        {"name": "ortho_3x1333x771_fp32", "op": "orthogonalize", "batch": 3, "rows": 1333, "cols": 771, "type": "fp32", "pad": 5},
        # the hidden layer of the 16-worker configuration
        {"name": "ortho_16x1024x1024_bf16", "op": "orthogonalize", "batch": 16, "rows": 1024, "cols": 1024, "type": "bf16", "pad": 0},
        # the widest hidden layer of the 64-worker configuration, half of its workers
        {"name": "ortho_32x2048x2048_bf16", "op": "orthogonalize", "batch": 32, "rows": 2048, "cols": 2048, "type": "bf16", "pad": 0},
        # a router's 64 x 1024 weights in 8 workers, fp32 masters
        {"name": "muon_8x64x1024_fp32", "op": "muon", "batch": 8, "rows": 64, "cols": 1024, "type": "fp32", "nesterov": True},
        # a ragged fp32 layer of a few workers
        {"name": "muon_4x500x1900_fp32", "op": "muon", "batch": 4, "rows": 500, "cols": 1900, "type": "fp32", "nesterov": False},
        # the first hidden layer 1024 -> 2048 of the 64-worker configuration, half of its workers, bf16 weights
        {"name": "muon_32x2048x1024_bf16", "op": "muon", "batch": 32, "rows": 2048, "cols": 1024, "type": "bf16", "nesterov": True},
        # one token: a step whose batch has shrunk to nothing but latency
        {"name": "route_1x1x64_k8_bf16", "op": "route", "groups": 1, "tokens": 1, "experts": 64, "k": 8, "type": "bf16", "normalize": True, "padded": False},
        # an odd expert count and ragged sequences behind a mask
        {"name": "route_16x1777x100_k3_fp32", "op": "route", "groups": 16, "tokens": 1777, "experts": 100, "k": 3, "type": "fp32", "normalize": False, "padded": True},
        # 16 workers with 16384 tokens each, 128 experts
        {"name": "route_16x16384x128_k8_bf16", "op": "route", "groups": 16, "tokens": 16384, "experts": 128, "k": 8, "type": "bf16", "normalize": True, "padded": False},
        # the gradient at an ordinary minibatch
        {"name": "grad_16x1777x100_k3_fp32", "op": "route_grad", "groups": 16, "tokens": 1777, "experts": 100, "k": 3, "type": "fp32", "normalize": False, "padded": True},
        # the gradient of the large one
        {"name": "grad_16x16384x128_k8_bf16", "op": "route_grad", "groups": 16, "tokens": 16384, "experts": 128, "k": 8, "type": "bf16", "normalize": True, "padded": False},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["orthogonalize", "muon", "route", "route_grad"])
    kind = rng.choice(["fp32", "bf16", "fp16"])
    if op in ("orthogonalize", "muon"):
        rows, cols, batch = _log(rng, 8, 2600), _log(rng, 8, 2600), _log(rng, 1, 64)
        s, l = min(rows, cols), max(rows, cols)
        most = 2.0e12 / (3 if kind == "fp32" else 1)
        batch = max(1, min(batch, int(most / (5 * (3.0 * s * s * l + s ** 3)))))
        if op == "orthogonalize":
            return {"op": op, "batch": batch, "rows": rows, "cols": cols, "type": kind, "pad": rng.choice([0, 0, 1, 8, 24])}
        return {"op": op, "batch": batch, "rows": rows, "cols": cols, "type": rng.choice(["fp32", "bf16"]), "nesterov": rng.random() < 0.5}
    groups, experts = _log(rng, 1, 64), _log(rng, 4, 512)
    tokens = max(1, min(_log(rng, 1, 20000), 16 * 16384 * 128 // (groups * experts)))
    return {"op": op, "groups": groups, "tokens": tokens, "experts": experts, "k": min(experts, rng.randint(1, 8)), "type": kind,
            "normalize": rng.random() < 0.5, "padded": rng.random() < 0.4}


# ---- inputs -------------------------------------------------------------------------------------------------
def _gradient_like(g, batch, rows, cols, steps=24, samples=32, decay=0.95):
    """What a momentum buffer holds: the decayed sum of minibatch gradients dZ^T X, each of rank `samples`; its
    spectrum falls off, and sides beyond steps * samples are rank deficient."""
    dz = torch.randn(batch, rows, steps * samples, generator=g, device=DEVICE)
    dz *= (decay ** torch.arange(steps, device=DEVICE, dtype=torch.float32)).repeat_interleave(samples)
    x = torch.randn(batch, steps * samples, cols, generator=g, device=DEVICE).relu_()
    return torch.bmm(dz, x).div_(samples)


def _wider(m, pad):
    """The matrices as the left columns of rows that are `pad` elements longer."""
    if not pad:
        return m
    big = torch.zeros(m.shape[0], m.shape[1], m.shape[2] + pad, dtype=m.dtype, device=m.device)
    big[:, :, :m.shape[2]] = m
    return big[:, :, :m.shape[2]]


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    op, kind = case["op"], TYPES[case["type"]]
    if op == "orthogonalize":
        m = _gradient_like(g, case["batch"], case["rows"], case["cols"]).to(kind)
        return {"op": op, "G": _wider(m, case["pad"]), "out": torch.empty_like(m)}
    if op == "muon":
        b, r, c = case["batch"], case["rows"], case["cols"]
        v = _gradient_like(g, b, r, c, steps=23).mul_(0.95)
        grad = _gradient_like(g, b, r, c, steps=1).to(kind)
        w = torch.randn(b, r, c, generator=g, device=DEVICE).div_(math.sqrt(c)).to(kind)
        return {"op": op, "W": w, "V": v, "G": grad, "lr": 0.02, "mu": 0.95, "wd": 0.01, "nesterov": case["nesterov"],
                "scale": math.sqrt(max(1.0, r / c))}
    n, t, e, k = case["groups"], case["tokens"], case["experts"], case["k"]
    favour = torch.randn(n, 1, e, generator=g, device=DEVICE)      # some experts are asked for more often than others
    logits = (torch.randn(n, t, e, generator=g, device=DEVICE) * 1.5 + favour).to(kind)
    live = None
    if case["padded"]:                                            # sequences padded to a common length
        lengths = torch.randint(0, t + 1, (n, 1), generator=g, device=DEVICE)
        live = (torch.arange(t, device=DEVICE)[None, :] < lengths).to(torch.uint8)
    state = {"op": op, "logits": logits, "live": live, "k": k, "coef": 0.01, "normalize": case["normalize"]}
    if op == "route_grad":
        chosen = torch.sort(logits.float(), dim=-1, descending=True, stable=True).indices[..., :k]
        if live is not None:
            chosen = torch.where(live[..., None] != 0, chosen, -1)
        state["experts"] = chosen.to(torch.int32).contiguous()
        state["counts"] = _count(chosen, e)
        # as under a loss scale: no gradient falls below what 16 bits hold, and both parts of it count
        state["dweights"] = torch.randn(n, t, k, generator=g, device=DEVICE)
        state["dloss"] = (torch.rand(n, generator=g, device=DEVICE) + 0.5) * (10.0 * t)
    return state


def _count(chosen, e):
    """How often each expert was chosen, [groups, e]; entries of -1 are not counted."""
    n = chosen.shape[0]
    at = torch.where(chosen < 0, e, chosen).reshape(n, -1).long()
    return torch.zeros(n, e + 1, dtype=torch.int64, device=chosen.device).scatter_add_(1, at, torch.ones_like(at))[:, :e].to(torch.int32).contiguous()


# ---- plain forms --------------------------------------------------------------------------------------------
def _newton_schulz(g, steps=5, eps=1e-7):
    a, b, c = COEFS
    norm = g.double().square().sum((1, 2), keepdim=True).sqrt()   # a sum of millions of squares
    x = (g.double() / (norm + eps)).float()
    tall = x.shape[1] > x.shape[2]
    if tall:
        x = x.mT
    for _ in range(steps):
        s = x @ x.mT
        x = a * x + (b * s + c * (s @ s)) @ x
    return x.mT if tall else x


def _softmax(x):
    e = (x - x.max(-1, keepdim=True).values).exp()
    return e / e.sum(-1, keepdim=True)


def _route(s):
    x, live, k = s["logits"].float(), s["live"], s["k"]
    n, t, e = x.shape
    p = _softmax(x)
    chosen = torch.sort(x, dim=-1, descending=True, stable=True).indices[..., :k]
    w = p.gather(-1, chosen)
    if s["normalize"]:
        w = w / w.sum(-1, keepdim=True)
    if live is not None:
        on = live[..., None] != 0
        chosen, w, p = torch.where(on, chosen, -1), torch.where(on, w, 0.0), torch.where(on, p, 0.0)
        tokens = live.float().sum(1, keepdim=True)
    else:
        tokens = torch.full((n, 1), float(t), device=x.device)
    counts = _count(chosen, e)
    mean = p.double().sum(1).float() / tokens.clamp(min=1)
    loss = s["coef"] * e * (counts.float() / (k * tokens.clamp(min=1)) * mean).sum(1)
    return chosen.to(torch.int32), w, counts, mean, loss


def _route_grad(s):
    x, live, k = s["logits"].float(), s["live"], s["k"]
    n, t, e = x.shape
    p = _softmax(x)
    tokens = live.float().sum(1, keepdim=True).clamp(min=1) if live is not None else torch.full((n, 1), float(t), device=x.device)
    h = (s["dloss"][:, None] * s["coef"] * e / tokens * (s["counts"].float() / (k * tokens)))[:, None, :].expand(n, t, e)
    chosen = s["experts"].long().clamp(min=0)
    dw = s["dweights"]
    if s["normalize"]:
        picked = p.gather(-1, chosen)
        total = picked.sum(-1, keepdim=True)
        dw = (dw - (dw * picked).sum(-1, keepdim=True) / total) / total
    h = h.scatter_add(-1, chosen, dw)
    d = p * (h - (p * h).sum(-1, keepdim=True))
    if live is not None:
        d = torch.where(live[..., None] != 0, d, 0.0)
    return d.to(s["logits"].dtype)


# ---- one pass -----------------------------------------------------------------------------------------------
def run(state):
    op = state["op"]
    if own:
        return _run_own(state)
    if op == "orthogonalize":
        return _newton_schulz(state["G"]).to(state["G"].dtype)
    if op == "muon":
        g, v, w, mu = state["G"].float(), state["V"], state["W"], state["mu"]
        v.mul_(mu).add_(g)
        u = g + mu * v if state["nesterov"] else v
        o = _newton_schulz(u)
        w.copy_((1.0 - state["lr"] * state["wd"]) * w.float() - state["lr"] * state["scale"] * o)
        return {"W": w, "V": v}
    if op == "route":
        return _route(state)
    return _route_grad(state)


def _run_own(state):
    from paper_1807_06629_b200 import binding as b
    op = state["op"]
    if op == "orthogonalize":
        if "work" not in state:
            state["work"] = b.orthogonalize_workspace(state["G"])
        return b.prsgd_orthogonalize(state["G"], out=state["out"], workspace=state["work"])
    if op == "muon":
        if "work" not in state:
            state["work"] = b.muon_workspace(state["W"])
        b.prsgd_muon_step(state["W"], state["V"], state["G"], state["lr"], mu=state["mu"], nesterov=state["nesterov"],
                          weight_decay=state["wd"], scale=state["scale"], workspace=state["work"])
        return {"W": state["W"], "V": state["V"]}
    if op == "route":
        if "work" not in state:
            state["work"] = b.route_workspace(state["logits"])
            state["outs"] = b.route_outputs(state["logits"], state["k"])
        return b.prsgd_route(state["logits"], state["k"], state["coef"], normalize=state["normalize"], live=state["live"],
                             out=state["outs"], workspace=state["work"])
    if "out" not in state:
        state["out"] = torch.empty_like(state["logits"])
    return b.prsgd_route_grad(state["logits"], state["experts"], state["counts"], state["coef"], normalize=state["normalize"],
                              live=state["live"], dweights=state["dweights"], dloss=state["dloss"], out=state["out"])


# ---- what a pass cannot do without --------------------------------------------------------------------------
def work(case):
    size = TYPES[case["type"]].itemsize
    if case["op"] in ("orthogonalize", "muon"):
        b, r, c = case["batch"], case["rows"], case["cols"]
        s, l = min(r, c), max(r, c)
        # per step: X X^T and its square are symmetric, half of each is enough
        flops = b * 5.0 * (s * (s + 1.0) * l + s * (s + 1.0) * s + 2.0 * s * s * l)
        each = 2 * size if case["op"] == "orthogonalize" else 3 * size + 8       # G, out | G, W twice, V twice
        return {"bytes": float(b * r * c * each), "flops": flops}
    n, t, e, k = case["groups"], case["tokens"], case["experts"], case["k"]
    mask = n * t if case["padded"] else 0
    if case["op"] == "route":
        return {"bytes": float(n * t * (e * size + 8 * k) + mask + n * (8 * e + 4)), "flops": float(n * t * e * 5)}
    return {"bytes": float(n * t * (2 * e * size + 8 * k) + mask + n * (4 * e + 4)), "flops": float(n * t * e * 8)}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------
def _exact_newton_schulz(g):
    a, b, c = COEFS
    x = g / (torch.linalg.vector_norm(g, dim=(1, 2), keepdim=True) + 1e-7)
    for _ in range(5):                                            # a X + S (b X + c S X), S on the short side
        if x.shape[1] <= x.shape[2]:
            s = torch.einsum("bij,bkj->bik", x, x)
            x = a * x + s @ (b * x + c * (s @ x))
        else:
            s = torch.einsum("bji,bjk->bik", x, x)
            x = a * x + (b * x + c * (x @ s)) @ s
    return x


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "orthogonalize":
        return _exact_newton_schulz(s["G"].double())
    if case["op"] == "muon":
        g = s["G"].double()
        v = s["mu"] * s["V"].double() + g
        o = _exact_newton_schulz(g + s["mu"] * v if s["nesterov"] else v)
        return {"W": s["W"].double() * (1.0 - s["lr"] * s["wd"]) - s["lr"] * s["scale"] * o, "V": v}
    x, k = s["logits"].double(), s["k"]
    n, t, e = x.shape
    on = s["live"].bool() if s["live"] is not None else torch.ones(n, t, dtype=torch.bool, device=x.device)
    many = on.sum(1).clamp(min=1).double()
    if case["op"] == "route":
        p = torch.exp(x - torch.logsumexp(x, -1, keepdim=True))
        values, at = torch.sort(x, dim=-1, descending=True, stable=True)
        at = at[..., :k]
        w = torch.exp(values[..., :k] - torch.logsumexp(values[..., :k] if s["normalize"] else values, -1, keepdim=True))
        share = torch.stack([(torch.nn.functional.one_hot(at[i][on[i]], e)).sum((0, 1)) if on[i].any() else torch.zeros(e, dtype=torch.int64, device=x.device)
                             for i in range(n)]).double()
        mean = (p * on[..., None]).sum(1) / many[:, None]
        loss = s["coef"] * e * (share / (k * many[:, None]) * mean).sum(1)
        return None, w * on[..., None], None, mean, loss
    x.requires_grad_(True)                                        # the gradient by differentiating the definition
    logp = torch.log_softmax(x, -1)
    mean = (logp.exp() * on[..., None]).sum(1) / many[:, None]
    loss = s["coef"] * e * (s["counts"].double() / (k * many[:, None]) * mean).sum(1)
    picked = logp.gather(-1, s["experts"].long().clamp(min=0))
    w = torch.softmax(picked, -1) if s["normalize"] else picked.exp()
    total = (loss * s["dloss"].double()).sum() + (w * on[..., None] * s["dweights"].double()).sum()
    return torch.autograd.grad(total, x)[0]
