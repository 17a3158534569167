"""Cases of the operators at the two ends of stacked workers' language models: the lookup of token embeddings and its
gradient by sorted tokens, dropout from a counter-based generator, and the softmax cross entropy over a vocabulary with its
gradient, whose logits are never kept.  Every operator is written here in its plain form (elementary torch operations in
fp32) and as the call of the library that computes the same."""
import math

import torch

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
DEVICE = "cuda:0"


# ---- cases --------------------------------------------------------------------------------------------------
def listed():
    return [
        # one token of one worker: latency
        {"name": "embed_1x1_v32000_d1024_bf16", "op": "embed", "groups": 1, "tokens": 1, "vocab": 32000, "dim": 1024, "type": "bf16", "out": "bf16", "padded": False},
        # a batch of long sequences in four workers, an odd vocabulary
        {"name": "embed_4x8192_v50257_d2048_bf16", "op": "embed", "groups": 4, "tokens": 8192, "vocab": 50257, "dim": 2048, "type": "bf16", "out": "bf16", "padded": True},
        # a small worker's fp32 table, odd sides, gradient of the whole table
        {"name": "embed_grad_2x500_v1000_d100_fp32", "op": "embed_grad", "groups": 2, "tokens": 500, "vocab": 1000, "dim": 100, "type": "fp32", "out": "fp32", "padded": True, "accumulate": False},
        # the batch above, added to the fp32 gradient that the class layer's share of a tied table has begun
        {"name": "embed_grad_4x8192_v50257_d2048_bf16", "op": "embed_grad", "groups": 4, "tokens": 8192, "vocab": 50257, "dim": 2048, "type": "bf16", "out": "fp32", "padded": True, "accumulate": True},
        # a minibatch of 32 rows, odd width
        {"name": "dropout_1x32x1001_fp32", "op": "dropout", "groups": 1, "rows": 32, "cols": 1001, "type": "fp32", "residual": False, "p": 0.5},
        # the hidden states of 16 workers with their residual stream
        {"name": "dropout_16x4096x2048_bf16", "op": "dropout", "groups": 16, "rows": 4096, "cols": 2048, "type": "bf16", "residual": True, "p": 0.1},
        # one token's loss: the weights are read once
        {"name": "loss_1x1_v32000_d1024_bf16", "op": "loss", "groups": 1, "tokens": 1, "vocab": 32000, "dim": 1024, "type": "bf16", "padded": False},
        # ragged sequences of 16 small fp32 workers, odd sizes, tokens without a label among them
        {"name": "loss_16x777_v1003_d500_fp32", "op": "loss", "groups": 16, "tokens": 777, "vocab": 1003, "dim": 500, "type": "fp32", "padded": True},
        # long sequences of one worker over a large vocabulary
        {"name": "loss_1x16384_v131072_d2048_bf16", "op": "loss", "groups": 1, "tokens": 16384, "vocab": 131072, "dim": 2048, "type": "bf16", "padded": False},
        # a minibatch of 64 in 16 workers over a thousand classes
        {"name": "loss_grad_16x64_v1000_d1024_fp16", "op": "loss_grad", "groups": 16, "tokens": 64, "vocab": 1000, "dim": 1024, "type": "fp16", "padded": False, "dlse": False},
        # four workers whose prompts carry no label; odd vocabulary, rows of 1000
        {"name": "loss_grad_4x2000_v32003_d1000_bf16", "op": "loss_grad", "groups": 4, "tokens": 2000, "vocab": 32003, "dim": 1000, "type": "bf16", "padded": True, "dlse": True},
        # a large step of one worker
        {"name": "loss_grad_1x8192_v65536_d2048_bf16", "op": "loss_grad", "groups": 1, "tokens": 8192, "vocab": 65536, "dim": 2048, "type": "bf16", "padded": False, "dlse": False},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["embed", "embed_grad", "dropout", "loss", "loss_grad"])
    kind = rng.choice(["fp32", "bf16", "fp16"])
    groups = _log(rng, 1, 32)
    if op == "dropout":
        cols = _log(rng, 30, 8200)
        rows = max(1, min(_log(rng, 1, 20000), 16 * 4096 * 2048 // (groups * cols) // (2 if kind == "fp32" else 1)))
        return {"op": op, "groups": groups, "rows": rows, "cols": cols, "type": kind, "residual": rng.random() < 0.5,
                "p": rng.choice([0.1, 0.2, 0.5, round(rng.uniform(0.01, 0.9), 3)])}
    dim = rng.choice([_log(rng, 32, 2100), 8 * _log(rng, 4, 260)])
    if op in ("embed", "embed_grad"):
        vocab = max(16, min(_log(rng, 100, 130000), 4 * 50257 * 2048 // (groups * dim)))
        tokens = max(1, min(_log(rng, 1, 20000), 4 * 8192 * 2048 // (groups * dim)))
        case = {"op": op, "groups": groups, "tokens": tokens, "vocab": vocab, "dim": dim, "type": kind,
                "out": rng.choice([kind, "fp32"]), "padded": rng.random() < 0.5}
        if op == "embed_grad":
            case["accumulate"] = rng.random() < 0.5
        return case
    most = 16384 * 131072 * 2048 if op == "loss" else 8192 * 65536 * 2048
    if kind == "fp32":
        most //= 4
    vocab = max(16, min(_log(rng, 100, 131000), 2 ** 29 // (groups * dim)))
    tokens = max(1, min(_log(rng, 1, 17000), most // (groups * dim * vocab)))
    case = {"op": op, "groups": groups, "tokens": tokens, "vocab": vocab, "dim": dim, "type": kind, "padded": rng.random() < 0.5}
    if op == "loss_grad":
        case["dlse"] = rng.random() < 0.5
    return case


# ---- inputs -------------------------------------------------------------------------------------------------
def _tokens(g, groups, tokens, vocab, padded):
    """Token ids as in text, the id's rank in frequency: p(id) = log((id + 2) / (id + 1)) / log(vocab + 1); padded: sequences that
    end early, -1 behind their end."""
    u = torch.rand(groups, tokens, generator=g, device=DEVICE, dtype=torch.float64)
    ids = ((vocab + 1.0) ** u).floor().long().sub_(1).clamp_(0, vocab - 1).to(torch.int32)
    if padded:
        length = torch.randint(0, tokens + 1, (groups, 1), generator=g, device=DEVICE)
        ids[torch.arange(tokens, device=DEVICE)[None, :] >= length] = -1
    return ids


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEVICE)


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    op, kind, n = case["op"], TYPES[case["type"]], case["groups"]
    if op == "dropout":
        shape = (n, case["rows"], case["cols"])
        return {"op": op, "x": _randn(g, *shape).to(kind), "residual": _randn(g, *shape).to(kind) if case["residual"] else None,
                "p": case["p"], "seed": 0x9E3779B97F4A7C15 * (seed + 1) % 2 ** 64, "step": 1000 + seed % 1000}
    t, v, d = case["tokens"], case["vocab"], case["dim"]
    ids = _tokens(g, n, t, v, case["padded"])
    if op == "embed":
        return {"op": op, "table": _randn(g, n, v, d).to(kind), "ids": ids, "scale": math.sqrt(d), "dtype": TYPES[case["out"]]}
    if op == "embed_grad":
        begun = _randn(g, n, v, d).to(TYPES[case["out"]]) if case["accumulate"] else torch.empty(n, v, d, dtype=TYPES[case["out"]], device=DEVICE)
        return {"op": op, "dout": _randn(g, n, t, d).to(kind), "ids": ids, "scale": 0.5, "dtable": begun, "accumulate": case["accumulate"]}
    # logits of a spread of 1.5 between classes; what a token's label gets beyond them is what the worker has learnt of it
    W = (_randn(g, n, v, d) * (1.5 / math.sqrt(d))).to(kind)
    H = _randn(g, n, t, d)
    for i in range(n):
        H[i] += 4.0 * torch.rand(t, 1, generator=g, device=DEVICE) * W[i][ids[i].clamp(min=0).long()].float()
    H = H.to(kind)
    state = {"op": op, "H": H, "W": W, "labels": ids}
    if op == "loss_grad":
        state["stats"] = torch.stack([_stats(H[i].float(), W[i].float()) for i in range(n)])
        # as under a loss scale: no gradient falls below what 16 bits hold
        state["dloss"] = torch.rand(n, t, generator=g, device=DEVICE) + 0.5
        # of a penalty on the squared logarithm of the softmax's denominator
        state["dlse"] = 2e-3 * state["stats"].sum(-1) * state["dloss"] if case["dlse"] else None
    return state


def _stats(H, W):
    """Largest logit and logarithm of the sum of e^(z - largest) of every token, [tokens, 2]."""
    out = torch.empty(H.shape[0], 2, device=H.device)
    for at in range(0, H.shape[0], 2048):
        z = H[at:at + 2048] @ W.mT
        m = z.max(-1, keepdim=True).values
        out[at:at + 2048, 0] = m[:, 0]
        out[at:at + 2048, 1] = (z - m).exp_().sum(-1).log()
    return out


# ---- plain forms --------------------------------------------------------------------------------------------
def _philox(c, key):
    """Ten rounds of Philox4x32 on four int64 tensors of 32-bit words."""
    low = 0xFFFFFFFF
    k0, k1 = key & low, key >> 32
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57                 # (modulo 2^64, whose upper half the shift and mask give)
        c = (((b >> 32) & low) ^ c[1] ^ k0, b & low, ((a >> 32) & low) ^ c[3] ^ k1, a & low)
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return c


def _keep(s):
    """Which elements stay: element c of a row takes 16 bits, the (c % 8)th of the generator's output at the counter
    (c / 8, row, group, step); it goes when they are below round(65536 p)."""
    n, r, c = s["x"].shape
    blocks = (c + 7) // 8
    at = lambda m, shape: torch.arange(m, device=DEVICE).view(shape).expand(n, r, blocks)
    w = _philox((at(blocks, (1, 1, -1)), at(r, (1, -1, 1)), at(n, (-1, 1, 1)), torch.full((n, r, blocks), s["step"] & 0xFFFFFFFF, device=DEVICE)), s["seed"])
    bits = torch.stack([h for x in w for h in (x & 0xFFFF, x >> 16)], -1).reshape(n, r, blocks * 8)[:, :, :c]
    return bits >= round(s["p"] * 65536)


def _dropout(s):
    scale = 65536.0 / (65536.0 - round(s["p"] * 65536))
    y = torch.where(_keep(s), s["x"].float() * scale, 0.0)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(s["x"].dtype)


def _embed(s):
    table, ids = s["table"], s["ids"]
    rows = torch.stack([table[i][ids[i].clamp(min=0).long()] for i in range(ids.shape[0])])
    return torch.where(ids[..., None] >= 0, rows.float() * s["scale"], 0.0).to(s["dtype"])


def _embed_grad(s):
    out = s["dtable"]
    for i in range(out.shape[0]):
        live = s["ids"][i] >= 0
        total = torch.zeros(out.shape[1], out.shape[2], dtype=torch.float64, device=DEVICE)     # (a frequent token's sum is long)
        total.index_add_(0, s["ids"][i][live].long(), s["dout"][i][live].double())
        total = (total * s["scale"]).float()
        out[i].copy_(out[i].float() + total if s["accumulate"] else total)
    return out


def _loss(s):
    losses, stats = [], []
    for H, W, y in zip(s["H"], s["W"], s["labels"]):
        z = H.float() @ W.float().mT
        m = z.max(-1).values
        log_sum = (z - m[:, None]).exp().sum(-1).log()
        live = y >= 0
        losses.append(torch.where(live, log_sum + (m - z.gather(-1, y.clamp(min=0).long()[:, None])[:, 0]), 0.0))
        stats.append(torch.where(live[:, None], torch.stack([m, log_sum], -1), 0.0))
    return torch.stack(losses), torch.stack(stats)


def _loss_grad(s):
    dH, dW = torch.empty_like(s["H"]), torch.empty_like(s["W"])
    for i in range(dH.shape[0]):
        H, W, y = s["H"][i].float(), s["W"][i].float(), s["labels"][i]
        live = y >= 0
        dloss = torch.where(live, s["dloss"][i], 0.0)
        both = dloss if s["dlse"] is None else dloss + torch.where(live, s["dlse"][i], 0.0)
        p = ((H @ W.mT - s["stats"][i][:, :1]) - s["stats"][i][:, 1:]).exp()
        p = p.mul_(both[:, None])
        p.scatter_add_(1, y.clamp(min=0).long()[:, None], -dloss[:, None])
        dH[i].copy_(p @ W)
        dW[i].copy_(p.mT @ H)
    return {"dH": dH, "dW": dW}


# ---- one pass -----------------------------------------------------------------------------------------------
def run(state):
    if own:
        return _run_own(state)
    return {"embed": _embed, "embed_grad": _embed_grad, "dropout": _dropout, "loss": _loss, "loss_grad": _loss_grad}[state["op"]](state)


def _run_own(s):
    from paper_1807_06629_b200 import binding as b
    op = s["op"]
    if op == "dropout":
        if "out" not in s:
            s["out"] = torch.empty_like(s["x"])
        return b.prsgd_dropout(s["x"], s["p"], s["seed"], step=s["step"], residual=s["residual"], out=s["out"])
    if op == "embed":
        if "out" not in s:
            s["out"] = torch.empty(*s["ids"].shape, s["table"].shape[-1], dtype=s["dtype"], device=s["table"].device)
        return b.prsgd_embed(s["table"], s["ids"], scale=s["scale"], out=s["out"])
    if op == "embed_grad":
        if "work" not in s:
            s["work"] = b.embed_grad_workspace(s["dout"], s["dtable"])
        return b.prsgd_embed_grad(s["dout"], s["ids"], s["dtable"], scale=s["scale"], accumulate=s["accumulate"], workspace=s["work"])
    if op == "loss":
        if "work" not in s:
            s["work"] = b.vocab_loss_workspace(s["H"], s["W"])
            s["out"] = b.vocab_loss_outputs(s["H"])
        return b.prsgd_vocab_loss(s["H"], s["W"], s["labels"], out=s["out"], workspace=s["work"])
    if "work" not in s:
        s["work"] = b.vocab_loss_grad_workspace(s["H"], s["W"])
        s["dH"], s["dW"] = torch.empty_like(s["H"]), torch.empty_like(s["W"])
    b.prsgd_vocab_loss_grad(s["H"], s["W"], s["labels"], s["stats"], dloss=s["dloss"], dlse=s["dlse"], dH=s["dH"], dW=s["dW"], workspace=s["work"])
    return {"dH": s["dH"], "dW": s["dW"]}


# ---- what a pass cannot do without --------------------------------------------------------------------------
def _distinct(tokens, vocab):
    """Expected number of different ids among that many tokens."""
    v = torch.arange(vocab, dtype=torch.float64)
    return float((1.0 - (1.0 - torch.log((v + 2.0) / (v + 1.0)) / math.log(vocab + 1.0)) ** tokens).sum())


def work(case):
    size, n, op = TYPES[case["type"]].itemsize, case["groups"], case["op"]
    if op == "dropout":
        count = n * case["rows"] * case["cols"]
        return {"bytes": float(count * size * (3 if case["residual"] else 2)), "flops": float(count * (2 if case["residual"] else 1))}
    t, v, d = case["tokens"], case["vocab"], case["dim"]
    live = t * (0.5 if case["padded"] else 1.0)                     # (sequences end anywhere)
    if op == "embed":
        return {"bytes": n * (_distinct(live, v) * d * size + t * (d * TYPES[case["out"]].itemsize + 4.0)), "flops": n * live * d}
    if op == "embed_grad":
        rows = 2.0 * _distinct(live, v) if case["accumulate"] else float(v)
        return {"bytes": n * (live * d * size + 4.0 * t + rows * d * TYPES[case["out"]].itemsize), "flops": n * live * d}
    if op == "loss":
        return {"bytes": n * (live * d * size + v * d * size + t * 16.0), "flops": n * 2.0 * live * v * d}
    # logits again, and a product of the same size for each gradient
    return {"bytes": n * ((live + t) * d * size + 2.0 * v * d * size + t * (20.0 if case["dlse"] else 16.0)), "flops": n * 6.0 * live * v * d}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------
def _times(a, b):
    """High and low words of a product of 32-bit words, by halves of 16 bits."""
    b1, b0 = b >> 16, b & 0xFFFF
    a1, a0 = a >> 16, a & 0xFFFF
    mid = a1 * b0 + ((a0 * b0) >> 16)
    side = a0 * b1 + (mid & 0xFFFF)
    return a1 * b1 + (mid >> 16) + (side >> 16), ((side & 0xFFFF) << 16) | ((a0 * b0) & 0xFFFF)


def _exact_keep(case, s, group):
    rows, cols = case["rows"], case["cols"]
    width = -(-cols // 8)
    x0 = torch.arange(width, device=DEVICE).repeat(rows)
    x1 = torch.arange(rows, device=DEVICE).repeat_interleave(width)
    x2, x3 = torch.full_like(x0, group), torch.full_like(x0, s["step"] % 2 ** 32)
    for r in range(10):
        ka, kb = (s["seed"] % 2 ** 32 + r * 0x9E3779B9) % 2 ** 32, (s["seed"] // 2 ** 32 + r * 0xBB67AE85) % 2 ** 32
        h0, l0 = _times(x0, 0xD2511F53)
        h1, l1 = _times(x2, 0xCD9E8D57)
        x0, x1, x2, x3 = h1 ^ x1 ^ ka, l1, h0 ^ x3 ^ kb, l0
    gone = torch.empty(rows * width, 8, dtype=torch.bool, device=DEVICE)
    for j, word in enumerate((x0, x1, x2, x3)):
        gone[:, 2 * j] = word % 65536 < round(case["p"] * 65536)
        gone[:, 2 * j + 1] = word // 65536 < round(case["p"] * 65536)
    return ~gone.view(rows, width * 8)[:, :cols]


def exact(case, seed):
    s = prepare(case, seed)
    op, n = case["op"], case["groups"]
    if op == "dropout":
        left = 1.0 - round(case["p"] * 65536) / 65536.0
        y = torch.stack([s["x"][i].double() * _exact_keep(case, s, i) / left for i in range(n)])
        return y if s["residual"] is None else y + s["residual"].double()
    ids = s["ids"] if op in ("embed", "embed_grad") else s["labels"]
    on = ids != -1
    if op == "embed":
        out = torch.zeros(n, case["tokens"], case["dim"], dtype=torch.float64, device=DEVICE)
        for i in range(n):
            out[i, on[i]] = s["table"][i].index_select(0, ids[i, on[i]]).double() * s["scale"]
        return out
    if op == "embed_grad":
        out = s["dtable"].double() if case["accumulate"] else torch.zeros(s["dtable"].shape, dtype=torch.float64, device=DEVICE)
        for i in range(n):
            order = torch.argsort(ids[i], stable=True)
            order = order[on[i][order]]
            if order.numel() == 0:
                continue
            which, many = torch.unique_consecutive(ids[i][order], return_counts=True)
            out[i, which.long()] += s["scale"] * torch.segment_reduce(s["dout"][i][order].double(), "sum", lengths=many, axis=0)
        return out
    if op == "loss":
        loss = torch.zeros(n, case["tokens"], dtype=torch.float64, device=DEVICE)
        stats = torch.zeros(n, case["tokens"], 2, dtype=torch.float64, device=DEVICE)
        for i in range(n):
            W = s["W"][i].double()
            for at in on[i].nonzero()[:, 0].split(2048):
                z = s["H"][i, at].double() @ W.T
                lse = torch.logsumexp(z, 1)
                loss[i, at] = lse - z.gather(1, ids[i, at, None].long())[:, 0]
                stats[i, at, 0] = z.amax(1)
                stats[i, at, 1] = lse - stats[i, at, 0]
        return loss, stats
    dH = torch.zeros(s["H"].shape, dtype=torch.float64, device=DEVICE)
    dW = torch.zeros(s["W"].shape, dtype=torch.float64, device=DEVICE)
    for i in range(n):
        W, st = s["W"][i].double(), s["stats"][i].double()
        for at in on[i].nonzero()[:, 0].split(2048):
            H = s["H"][i, at].double()
            dl = s["dloss"][i, at].double()
            dn = dl if s["dlse"] is None else dl + s["dlse"][i, at].double()
            G = torch.exp(H @ W.T - st[at].sum(1, keepdim=True)) * dn[:, None]
            G[torch.arange(at.numel(), device=DEVICE), ids[i, at].long()] -= dl
            dH[i, at] = G @ W
            dW[i] += G.T @ H
    return {"dH": dH, "dW": dW}
