"""The vocabulary loss and its gradient over weights of more than 2^31 elements and 2^32 bytes, in pieces against the formulas in 64 bits."""
import math

import pytest
import torch

from test_gpu_language import BF16, F32, U, b, check, gen, half, randn, z_error          # noqa: F401  (b: a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,T", [(BF16, 1), (BF16, 40), (F32, 2), (F32, 40)])
def test_weights_beyond_32_bits(b, dtype, T):
    """Tolerances as in test_gpu_language.py, with e_z of each token; dH's contraction is cut into sums of 16384 products at most, the 32 of them
    added in fp32."""
    V, D = (1 << 21) + 77, 1032
    W = torch.randn(1, V, D, generator=gen(600), device="cuda:0", dtype=dtype)
    W *= 2.0 ** -4
    H = randn(601, 1, T, D, dtype=dtype)
    y = torch.randint(0, V, (1, T), generator=gen(602), device="cuda:0").to(torch.int32)
    y[0, 0] = V - 1
    if T > 2:
        y[0, 1], y[0, 5] = 0, -1
    on = y[0] >= 0
    Hd = torch.where(on[:, None], H[0].double(), 0.0)
    spans = [(v, min(V, v + (1 << 18))) for v in range(0, V, 1 << 18)]
    top, total, label, ez = torch.full((T,), -math.inf, device="cuda:0", dtype=torch.float64), 0.0, 0.0, 0.0
    for v0, v1 in spans:
        z = Hd @ W[0, v0:v1].double().T
        m = torch.maximum(top, z.amax(1))
        total = total * (top - m).exp() + (z - m[:, None]).exp().sum(1)
        top = m
        mine = (y[0] >= v0) & (y[0] < v1)
        label = label + torch.where(mine, z.gather(1, (y[0].long() - v0).clamp(0, v1 - v0 - 1)[:, None])[:, 0], 0.0)
        ez = torch.maximum(z_error(Hd.to(dtype), W[0, v0:v1], D).amax(1), torch.as_tensor(ez, device="cuda:0"))
    log_sum = total.log()
    loss, stats = b.prsgd_vocab_loss(H, W, y)
    tol = 2 * ez + 2.0 ** -14 + 8 * U * (top.abs() + (log_sum + top - label).abs())
    check(loss[0], torch.where(on, log_sum + top - label, 0.0), tol)
    check(stats[0, :, 0], torch.where(on, top, 0.0), ez + 2 * U * top.abs())
    check(stats[0, :, 1], torch.where(on, log_sum, 0.0), tol)

    stats = torch.where(on[:, None], torch.stack([top, log_sum], -1), 0.0).float()[None]
    dloss = randn(603, 1, T)
    work = b.vocab_loss_grad_workspace(H, W)
    dH, dW = b.prsgd_vocab_loss_grad(H, W, y, stats, dloss=dloss, workspace=work)
    b.prsgd_work_status(work)
    dl = torch.where(on, dloss[0].double(), 0.0)
    hold = half(dtype) if dtype != F32 else 2.0 ** -21
    off = hold + 2 * ez[:, None] + 2.0 ** -20
    wH, mH, sums = 0.0, 0.0, 0.0
    for v0, v1 in spans:
        w = W[0, v0:v1].double()
        p = (Hd @ w.T - top[:, None] - log_sum[:, None]).exp() * on[:, None]
        hot = ((y[0].long()[:, None] - v0) == torch.arange(v1 - v0, device="cuda:0")) & on[:, None]
        G, A = dl[:, None] * (p - hot.double()), dl.abs()[:, None] * (p + hot)
        wH, mH, sums = wH + G @ w, mH + (off * A) @ w.abs() + 1032 * 2.0 ** -22 * (A @ w.abs()), sums + w.abs().sum(0)
        lost = 2.0 ** -37 * dl.abs().amax() * Hd.abs().sum(0)
        check(dW[0, v0:v1], G.T @ Hd, (A * (off + (T / 16 + 4) * 2.0 ** -22)).T @ Hd.abs() + lost + 2 * half(dtype) * (G.T @ Hd).abs())
    check(dH[0], wH, mH + 2.0 ** -20 * wH.abs() + 2.0 ** -38 * dl.abs()[:, None] * sums + half(dtype) * wH.abs())
