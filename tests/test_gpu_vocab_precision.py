"""Precision of the vocabulary loss and its gradient where the tests of test_gpu_language.py are too wide to see it: sums whose terms have
one sign, long contractions, means of signed errors."""
import math

import pytest
import torch

import language_reference as ref
from test_gpu_language import BF16, F16, F32, U, b, case, check, gen, half, randn, z_error          # noqa: F401  (b: a fixture)

pytestmark = pytest.mark.gpu


# ---- long contractions ----------------------------------------------------------------------------------------
# A tensor core cuts off what the running sum does not hold, towards zero: n products of one sign are off by (n / 16 + 4) 2^-22 of their sum at
# most.  Sums of up to 8192 products are formed at once, longer ones from sums of 4096 that are added in fp32 (one rounding each): the bound
# stops growing at 4096.
def one_sum(n):
    return (min(n, 8192) / 16 + 4) * 2.0 ** -22 if n <= 8192 else (4096 / 16 + 4) * 2.0 ** -22 + math.ceil(n / 4096) * U


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("dtype,out", [(BF16, F32), (F16, F32), (BF16, BF16), (F32, F32)])
@pytest.mark.parametrize("T", [8192, 8200, 131072])
def test_gradient_of_many_tokens(b, T, dtype, out, accumulate):
    """W = 0: p = 1 / V = 2^-8 for every class, which G's type holds, so that dW = 2^-8 sum_t H_t (dlse = 1, no dloss) and what is off
    is the sum alone (p itself: 2^-20).  H of one sign."""
    V, D = 256, 72
    H = (torch.rand(1, T, D, generator=gen(1), device="cuda:0").square() + 2.0 ** -6).to(dtype)
    W = torch.zeros(1, V, D, dtype=dtype, device="cuda:0")
    y = torch.zeros(1, T, dtype=torch.int32, device="cuda:0")
    stats = torch.tensor([0.0, math.log(V)], device="cuda:0").expand(1, T, 2).contiguous()
    before = (randn(2, 1, V, D) * T * 2.0 ** -9).to(out) if accumulate else None
    dW = before.clone() if accumulate else torch.full((1, V, D), float("nan"), dtype=out, device="cuda:0")
    work = b.vocab_loss_grad_workspace(H, W).fill_(0xFF)
    dH, _ = b.prsgd_vocab_loss_grad(H, W, y, stats, dlse=torch.ones(1, T, device="cuda:0"), dW=dW, accumulate=accumulate, workspace=work)
    b.prsgd_work_status(work)
    sums = (H.double().sum(1, keepdim=True) / V).expand(1, V, D)
    want = sums + before.double() if accumulate else sums
    hold = 2.0 ** -21 if dtype == F32 else 0.0                # (of pairs)
    check(dW, want, (one_sum(T) + 2.0 ** -20 + hold) * sums + (half(out) + 2 * U) * want.abs())
    assert (dH == 0).all()


def test_gradient_of_many_columns(b):
    """Logits that are sums of 65536 products of one sign: z = 20 for every class, p = 2^-8 e^(their error).  One rounding of G, two of dW's
    terms are exact."""
    T, V, D = 40, 256, 65536
    H = torch.ones(1, T, D, dtype=F16, device="cuda:0")
    row = ((torch.rand(D, generator=gen(3), device="cuda:0") + 0.5) * (20.0 / D)).to(F16)
    W = row.expand(1, V, D).contiguous()
    z = row.double().sum().item()
    y = torch.zeros(1, T, dtype=torch.int32, device="cuda:0")
    stats = torch.tensor([z, math.log(V)], device="cuda:0").expand(1, T, 2).contiguous()
    dW = torch.empty(1, V, D, device="cuda:0")
    dH, _ = b.prsgd_vocab_loss_grad(H, W, y, stats, dlse=torch.ones(1, T, device="cuda:0"), dW=dW)
    off = one_sum(D) * z + 2 * U * z + 2.0 ** -20 + half(F16)
    check(dW, torch.full_like(dW, T / V).double(), torch.tensor((off + one_sum(T)) * T / V, device="cuda:0"))
    want = row.double().expand(1, T, D)
    check(dH, want, (off + one_sum(V) + half(F16)) * want + 2.0 ** -25)


# ---- fp16: gradients of different sizes in one group ----------------------------------------------------------
@pytest.mark.parametrize("G,T,V,D", [(1, 60, 20000, 64), (2, 300, 2500, 100), (3, 70, 400, 1100), (1, 8300, 600, 40), (3, 4100, 300, 24)])
def test_fp16_gradients_of_any_size(b, G, T, V, D):
    """fp16: tokens whose dloss and dlse are up to 2^30 smaller than the group's largest (2^13), beside some without any: a token's row of dH
    is as good, relative to its own, as that of the largest.  A last column of ones in W makes that column of dH dlse_t: what G's smallest entries lose shows there.

    G: one rounding, and 2^-26 d_t (d = |dloss| + |dlse|) where fp16 has no more bits: its row is held such that d_t lies in [2, 2^14).  dW: the same
    with H's row, which is held in fp16 times d_t's share of the largest beyond 2^-12: 2^-25 of its unit, 2^-36 of the largest d_t a G of d_t."""
    H, W, y = case(130, G, T, V, D, F16, padded=T < 1000)
    W[..., -1] = 1.0
    size = 2.0 ** (13.0 - (torch.arange(T, device="cuda:0") % 31))
    dloss = (torch.rand(G, T, generator=gen(133), device="cuda:0") - 0.5) * 0.8 * size
    dlse = (0.5 + 0.5 * torch.rand(G, T, generator=gen(134), device="cuda:0")) * 0.5 * size
    dloss[:, 5::17], dlse[:, 5::17] = 0.0, 0.0
    stats = ref.vocab_loss(H, W, y)[1].float()
    dW = torch.full((G, V, D), float("nan"), device="cuda:0")
    work = b.vocab_loss_grad_workspace(H, W).fill_(0xFF)
    dH, _ = b.prsgd_vocab_loss_grad(H, W, y, stats, dloss=dloss, dlse=dlse, dW=dW, workspace=work)
    b.prsgd_work_status(work)
    wH, wW, mH, mW, A = ref.vocab_grad(H, W, y, dloss, dlse)
    on = ref.live_tokens(y, V)
    Hz, d = H.double().abs() * on[..., None], (dloss.abs() + dlse.abs()).double() * on
    top = d.amax(1)[:, None, None]
    ez = z_error(Hz, W, D).amax(-1, keepdim=True) + 4 * U * stats.double().abs().sum(-1, keepdim=True)
    off = lambda n: half(F16) + 2 * ez + 2.0 ** -20 + (n / 16 + 4) * 2.0 ** -22          # noqa: E731
    check(dH, wH, off(V) * mH + 2.0 ** -26 * d[..., None] * W.double().abs().sum(1, keepdim=True) + half(F16) * wH.abs() + 2.0 ** -25)
    share = (A / d.clamp(min=1e-300)[..., None]).sum(1)[..., None]
    check(dW, wW, (A * off(T)).mT @ Hz + 2.0 ** -37 * top * Hz.sum(1, keepdim=True) + 2.0 ** -36 * top * share + 2 * half(F32) * wW.abs())
    only = b.prsgd_vocab_loss_grad(H, W, y, stats, dloss=dloss, dlse=dlse, want_dW=False)[0]
    assert torch.equal(only, dH)


def test_fp16_gradients_beyond_a_floats_exponents(b):
    """Sizes whose quotient no float holds: the small ones' rows are theirs alone, the large ones' share of dW is not touched."""
    H, W, y = case(140, 1, 40, 300, 64, F16, padded=False)
    stats = ref.vocab_loss(H, W, y)[1].float()
    dloss = torch.full((1, 40), 2.0 ** 100, device="cuda:0")
    dloss[0, 20:] = 2.0 ** -60
    dW = torch.empty(1, 300, 64, device="cuda:0")
    b.prsgd_vocab_loss_grad(H, W, y, stats, dloss=dloss, dW=dW, want_dH=False)
    alone, large = torch.where(dloss > 1, y, -1), torch.empty_like(dW)
    b.prsgd_vocab_loss_grad(H, W, alone, stats, dloss=dloss, dW=large, want_dH=False)
    assert torch.isfinite(dW).all() and torch.equal(dW, large)
    dloss[0, 20:], dloss[0, :20] = 1.0, 2.0 ** 120
    want = b.prsgd_vocab_loss_grad(H, W, torch.where(dloss == 1, y, -1), stats, dloss=dloss)[0]
    got = b.prsgd_vocab_loss_grad(H, W, y, stats, dloss=dloss)[0]
    check(got[:, 20:], want[:, 20:].double(), 2.0 ** -9 * want[:, 20:].double().abs() + 2.0 ** -12)


@pytest.mark.parametrize("T", [70, 4200])
def test_fp16_gradients_captured(b, T):
    """Replays with other gradients and labels, whose sizes move what is held by its own size, give what direct calls do; so do two streams at once."""
    G, V, D = 2, 300, 24
    H, W, y = case(150, G, T, V, D, F16)
    stats = ref.vocab_loss(H, W, torch.where(y < 0, 0, y.clamp(max=V - 1)))[1].float()
    size = lambda n: 2.0 ** -(torch.arange(T, device="cuda:0") * (n + 1) % 40).float()          # noqa: E731
    dloss, labels = randn(153, G, T), y.clone()
    dH, dW, work = torch.empty_like(H), torch.empty_like(W), b.vocab_loss_grad_workspace(H, W)
    call = lambda: b.prsgd_vocab_loss_grad(H, W, labels, stats, dloss=dloss, dH=dH, dW=dW, workspace=work)          # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for n in range(3):
        dloss.copy_(randn(160 + n, G, T) * size(n))
        labels.copy_(y.roll(n, 1))
        dH.fill_(float("nan")), dW.fill_(float("nan"))
        graph.replay()
        want = b.prsgd_vocab_loss_grad(H, W, labels, stats, dloss=dloss)
        assert torch.equal(dH, want[0]) and torch.equal(dW, want[1]), n
    torch.cuda.synchronize()
    got = []
    for s in (torch.cuda.Stream(), torch.cuda.Stream()):
        with torch.cuda.stream(s):
            got.append(b.prsgd_vocab_loss_grad(H, W, labels, stats, dloss=dloss))
    torch.cuda.synchronize()
    for one in got:
        assert torch.equal(one[0], want[0]) and torch.equal(one[1], want[1])


# ---- fp32: the gradient's logits --------------------------------------------------------------------------------
@pytest.mark.parametrize("T,D", [(512, 2048), (40, 1000)])
def test_gradient_logits_are_good_to_fp32(b, T, D):
    """A column of ones in W makes that column of dH sum_v p_tv (dlse = 1, no dloss): off from 1 by the relative error of the softmax, which is the absolute one of the
    logits that make it up (here 10 to 20 of learnt tokens).  A logit is a sum of sums of 64 products, each cut off four times, when it holds 1/4, 2/4, 3/4 and 4/4 of its
    end, each time by 2^-22 of that at most (test_gpu_language.py) and by half as much on average: 2.5 x 2^-23 of it; dH sums of 256 products: 2^-21; pairs, exponential: 2^-21.
    Additions in fp32 have no sign.  (A logit as sums of 512 products: 32 times, 16.5 x 2^-23.)"""
    V = 1000
    H, W, y = case(170, 1, T, V, D, F32, padded=False, spread=1.5)
    H += 7.0 * W[0][y[0].long()]
    W[..., -1] = 1.0
    H[..., -1] = 0.0
    exact = ref.vocab_loss(H, W, y)[1]
    stats = exact.float()
    dH, _ = b.prsgd_vocab_loss_grad(H, W, y, stats, dlse=torch.ones(1, T, device="cuda:0"))
    want = (exact.sum(-1) - stats.double().sum(-1)).exp()    # (the stats' own rounding)
    off = ((dH[0, :, -1].double() - want[0])).mean().abs().item()
    z = exact[..., 0].abs().mean().item()
    assert z > 8 and off <= 2.5 * 2.0 ** -23 * z + 2.0 ** -20, (off, z)


# ---- statistics -----------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("D", [2048, 4000])
def test_statistics_are_good_to_fp32(b, D, dtype):
    """Largest logit and logarithm of the denominator of normal data: rms and mean of the signed error relative to their size.  Logits are sums of 512
    products, each cut off 32 times by 2^-24 of what it holds, half its end on average: 9.5e-7; one sum of D = 2048 is off by 1.9e-6, of 4000 by
    twice that."""
    T, V = 512, 3000
    H, W = randn(500, 1, T, D, dtype=dtype), (randn(501, 1, V, D) * (1.5 / math.sqrt(D))).to(dtype)
    y = torch.randint(0, V, (1, T), generator=gen(502), device="cuda:0").to(torch.int32)
    loss, stats = b.prsgd_vocab_loss(H, W, y)
    want, exact = ref.vocab_loss(H, W, y)
    for got, true in ((stats[..., 0], exact[..., 0]), (stats.double().sum(-1), exact.sum(-1)), (loss, want)):
        error = got.double() - true
        size = true.square().mean().sqrt()
        assert error.square().mean().sqrt() <= 1e-6 * size and error.mean().abs() <= 1e-6 * size, (error.square().mean().sqrt() / size, error.mean() / size)
