"""Precision of the vocabulary loss and its gradient where the tests of test_gpu_language.py are too wide to see it: sums whose terms have
one sign, long contractions, means of signed errors."""
import math

import pytest
import torch

import language_reference as ref
from test_gpu_language import BF16, F16, F32, U, b, check, gen, half, randn          # noqa: F401  (b: a fixture)

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
