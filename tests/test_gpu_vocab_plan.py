"""The vocabulary loss and its gradient at sizes whose plan has several tiles a task, several pieces and parts, and several sums a tile
(vocab_shapes.py; test_vocab_plan.py checks that they have), against the formulas in 64 bits; tolerances as in test_gpu_language.py."""
import pytest
import torch

import language_reference as ref
import vocab_shapes as shapes
from test_gpu_language import BF16, F16, F32, b, case, check_grad, check_loss, exact_stats, randn          # noqa: F401  (b: a fixture)

pytestmark = pytest.mark.gpu


def gradient(b, G, T, V, D, dtype, out, accumulate):
    """Several calls, of the same bits, none with an expired wait; the second of several groups has no label."""
    H, W, y = case(400, G, T, V, D, dtype)
    if G > 1:
        y[1] = -1
    stats = torch.cat([exact_stats(H[g:g + 1], W[g:g + 1], y[g:g + 1]) for g in range(G)])
    dloss, dlse = randn(403, G, T), randn(404, G, T) * 0.1
    before = randn(405, G, V, D, dtype=out) if accumulate else None
    work = b.vocab_loss_grad_workspace(H, W).fill_(0xFF)
    first = None
    for n in range(5):
        dW = before.clone() if accumulate else torch.full((G, V, D), float("nan"), dtype=out, device="cuda:0")
        got = b.prsgd_vocab_loss_grad(H, W, y, stats, dloss=dloss, dlse=dlse, dW=dW, accumulate=accumulate, workspace=work)
        b.prsgd_work_status(work)
        if first is None:
            first = got
        assert torch.equal(got[0], first[0]) and torch.equal(got[1], first[1]), n
    for g in range(G):
        one = slice(g, g + 1)
        check_grad((first[0][one], first[1][one]), H[one], W[one], y[one], dloss[one], dlse[one], before[one] if accumulate else None)
    if G > 1:
        assert torch.equal(first[1][1], before[1] if accumulate else torch.zeros_like(first[1][1])) and (first[0][1] == 0).all()


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("dtype,out", [(BF16, F32), (F16, F16), (F32, F32)])
@pytest.mark.parametrize("G,T,V,D", shapes.RUNS_OF_DW)
def test_gradient_of_several_tiles_a_task(b, G, T, V, D, dtype, out, accumulate):
    gradient(b, G, T, V, D, dtype, out, accumulate)


@pytest.mark.parametrize("dtype,out", [(BF16, F32), (F16, F16), (F32, F32)])
@pytest.mark.parametrize("G,T,V,D", shapes.PIECES)
def test_gradient_of_several_pieces_parts_and_columns(b, G, T, V, D, dtype, out):
    gradient(b, G, T, V, D, dtype, out, False)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("dtype,out", [(BF16, F32), (F16, F16)])
@pytest.mark.parametrize("G,T,V,D", shapes.LONG)
def test_gradient_of_cut_sums(b, G, T, V, D, dtype, out, accumulate):
    gradient(b, G, T, V, D, dtype, out, accumulate)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("G,T,V,D", shapes.RUNS_OF_LOSS)
def test_loss_of_several_tiles_a_task(b, G, T, V, D, dtype):
    H, W, y = case(410, G, T, V, D, dtype)
    if G > 1:
        y[1, T // 3:] = -1
    work = b.vocab_loss_workspace(H, W).fill_(0xFF)
    first = b.prsgd_vocab_loss(H, W, y, workspace=work)
    b.prsgd_work_status(work)
    for g in range(G):
        one = slice(g, g + 1)
        check_loss((first[0][one], first[1][one]), H[one], W[one], y[one])
    for n in range(5):
        got = b.prsgd_vocab_loss(H, W, y, workspace=work)
        b.prsgd_work_status(work)
        assert torch.equal(got[0], first[0]) and torch.equal(got[1], first[1]), n


@pytest.mark.parametrize("kind", ["dense", "odd"])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("G,T,V,D", shapes.FEW + shapes.NOT_FEW)
def test_loss_of_few_tokens(b, G, T, V, D, dtype, kind):
    H, W, y = case(420, G, T, V, D, dtype, kind)
    if G > 1:
        y[1] = -1
        H[1] = float("nan")
    work = b.vocab_loss_workspace(H, W).fill_(0xFF)
    got = b.prsgd_vocab_loss(H, W, y, workspace=work)
    b.prsgd_work_status(work)
    check_loss(got, torch.where(ref.live_tokens(y, V)[..., None], H, 0), W, y)
