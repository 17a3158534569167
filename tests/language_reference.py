"""Embedding, dropout and vocabulary cross entropy written from their formulas in 64 bits (torch, any device)."""
import numpy as np
import torch


def live_tokens(ids, vocab):
    return (ids >= 0) & (ids < vocab)


def embed(table, ids, scale=1.0):
    on = live_tokens(ids, table.shape[1])
    rows = torch.stack([table[g][ids[g].long().clamp(0, table.shape[1] - 1)].double() for g in range(table.shape[0])])
    return torch.where(on[..., None], rows * scale, 0.0)


def embed_grad(dout, ids, vocab, scale=1.0):
    """(gradient, sum of the magnitudes that were added, how many were) per table row."""
    G, T, D = dout.shape
    sums = torch.zeros(G, vocab, D, dtype=torch.float64, device=dout.device)
    mags, many = torch.zeros_like(sums), torch.zeros(G, vocab, dtype=torch.float64, device=dout.device)
    on = live_tokens(ids, vocab)
    for g in range(G):
        at, rows = ids[g][on[g]].long(), dout[g][on[g]].double()
        sums[g].index_add_(0, at, rows * scale)
        mags[g].index_add_(0, at, (rows * scale).abs())
        many[g].index_add_(0, at, torch.ones(at.numel(), dtype=torch.float64, device=dout.device))
    return sums, mags, many


def philox(counter, key):
    """Ten rounds of Philox4x32 on numpy uint64 arrays of 32-bit words."""
    low = np.uint64(0xFFFFFFFF)
    x = [np.asarray(c, dtype=np.uint64) for c in counter]
    k = [np.uint64(key & 0xFFFFFFFF), np.uint64(key >> 32)]
    for _ in range(10):
        a, b = x[0] * np.uint64(0xD2511F53), x[2] * np.uint64(0xCD9E8D57)
        x = [(b >> np.uint64(32)) ^ x[1] ^ k[0], b & low, (a >> np.uint64(32)) ^ x[3] ^ k[1], a & low]
        k = [(k[0] + np.uint64(0x9E3779B9)) & low, (k[1] + np.uint64(0xBB67AE85)) & low]
    return x


def dropout_keep(groups, rows, cols, p, seed, step=0, first_group=0):
    """bool [groups, rows, cols]: which elements stay."""
    blocks = (cols + 7) // 8
    g, r, b = np.meshgrid(np.arange(groups) + first_group, np.arange(rows), np.arange(blocks), indexing="ij")
    w = philox((b, r, g & 0xFFFFFFFF, np.full(b.shape, step & 0xFFFFFFFF)), seed)
    bits = np.stack([h for x in w for h in (x & np.uint64(0xFFFF), x >> np.uint64(16))], -1).reshape(groups, rows, blocks * 8)[..., :cols]
    return bits >= np.uint64(round(p * 65536))


def dropout(x, p, seed, step=0, first_group=0, residual=None):
    keep = torch.from_numpy(dropout_keep(*x.shape, p, seed, step, first_group)).to(x.device)
    y = torch.where(keep, x.double() * (65536.0 / (65536.0 - round(p * 65536))), 0.0)
    return y if residual is None else y + residual.double()


def logits(H, W):
    return H.double() @ W.double().mT


def vocab_loss(H, W, labels):
    on = live_tokens(labels, W.shape[1])
    z = torch.where(on[..., None], logits(torch.where(on[..., None], H, 0), W), 0.0)
    m = z.amax(-1)
    log_sum = (z - m[..., None]).exp().sum(-1).log()
    y = labels.long().clamp(0, W.shape[1] - 1)
    loss = log_sum + m - z.gather(-1, y[..., None])[..., 0]
    return torch.where(on, loss, 0.0), torch.where(on[..., None], torch.stack([m, log_sum], -1), 0.0)


def vocab_grad(H, W, labels, dloss=None, dlse=None):
    """(dH, dW, |G| |W|, |G|^T |H|, |G|), |G| = |dloss + dlse| p + |dloss| onehot: what the terms of a sum amount to."""
    V = W.shape[1]
    on = live_tokens(labels, V)
    zero = torch.zeros(labels.shape, dtype=torch.float64, device=H.device)
    dl = zero if dloss is None else torch.where(on, dloss.double(), zero)
    dn = dl if dlse is None else dl + torch.where(on, dlse.double(), zero)
    Hd = torch.where(on[..., None], H.double(), 0.0)
    p = torch.softmax(logits(Hd, W), -1)
    p = torch.where(on[..., None], p, 0.0)
    hot = torch.nn.functional.one_hot(labels.long().clamp(0, V - 1), V).double() * on[..., None]
    G = dn[..., None] * p - dl[..., None] * hot
    A = dn.abs()[..., None] * p + dl.abs()[..., None] * hot
    return G @ W.double(), G.mT @ Hd, A @ W.double().abs(), A.mT @ Hd.abs(), A
