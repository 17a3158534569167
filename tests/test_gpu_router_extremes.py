"""The router and its gradient on rows of very large logits, against the formulas in 64 bits (tests/operator_reference.py).

A row whose every logit is the type's lowest value, or any other number, has p = 1 / E: its experts are the first ones, and
only a row of -inf has none.  Tolerances: the exponent of a logit d below the largest is d log2e, rounded twice (2^-24 each) with a
constant off by 2^-26 of itself, so e^-d is off by d e^-d 2.3 2^-24 <= 6e-8, and ex2.approx adds 2^-22; the sum of E terms is made of at
most 32 in a row and 5 halvings, 37 2^-24 = 2.2e-6: below 3e-6 of a weight, itself at most 1.  Allowed 5e-6 for the weights and 1e-5
of the largest for the mean, a sum over at most 2^5 such rows by lanes.  A gradient p (h - sum p h): 2e-5 of the largest upstream
gradient times p, plus the half-step of its type."""
import pytest
import torch

import operator_reference as ref

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def b():
    from paper_1807_06629_b200 import _build
    _build.build_library()
    from paper_1807_06629_b200 import binding
    assert torch.cuda.is_available()
    return binding


def rows_of(dtype):
    top = torch.finfo(dtype).max
    big = (1e4, 6e4) if dtype == F16 else (1e9, 1e10, 1e12, 1e30)
    return [v for s in (-1.0, 1.0) for v in [s * x for x in big] + [s * top]]


def extremes(dtype, E):
    """Two groups: rows of one value each, rows with one logit away from the rest, ordinary rows between them; and the same again
    behind the type's lowest value in half of the places."""
    g = torch.Generator(device="cuda:0")
    g.manual_seed(7)
    low, rows = torch.finfo(dtype).min, []
    for v in rows_of(dtype):
        rows.append(torch.full((E,), v, device="cuda:0"))
        rows.append(torch.randn(E, generator=g, device="cuda:0"))
        one = torch.full((E,), v, device="cuda:0")
        one[E // 2] = v * 0.75
        rows.append(one)
    x = torch.stack(rows).to(dtype)
    half = x.clone()
    half[:, E // 3:] = low
    return torch.stack([x, half])


@pytest.mark.parametrize("normalize", [False, True])
@pytest.mark.parametrize("E,k", [(6, 2), (8, 8), (64, 8), (64, 9), (130, 4), (300, 1), (1000, 8), (40, 20)])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_route_of_very_large_logits(b, dtype, E, k, normalize):
    x = extremes(dtype, E)
    work = torch.full((b.prsgd_route_workspace_bytes(*x.shape),), 0xFF, dtype=torch.uint8, device="cuda:0")
    experts, weights, counts, mean, loss = b.prsgd_route(x, k, 0.01, normalize=normalize, workspace=work)
    want = ref.route(x, k, 0.01, normalize)
    assert torch.equal(experts.long(), want[0]) and torch.equal(counts.long(), want[2])
    assert (weights.double() - want[1]).abs().max() <= 5e-6
    assert (mean.double() - want[3]).abs().max() <= 1e-5 * want[3].max()
    assert ((loss.double() - want[4]).abs() <= 1e-5 * want[4].abs()).all()


def test_a_group_with_a_row_of_the_lowest_value_keeps_its_loss(b):
    """A token whose mask leaves nothing but fill values is one of many: the group's mean and loss stay numbers."""
    g = torch.Generator(device="cuda:0")
    g.manual_seed(8)
    for dtype in (F32, BF16, F16):
        x = torch.randn(3, 700, 64, generator=g, device="cuda:0").to(dtype)
        x[1, 300] = torch.finfo(dtype).min
        experts, weights, counts, mean, loss = b.prsgd_route(x, 8, 0.01)
        want = ref.route(x, 8, 0.01)
        assert torch.equal(experts.long(), want[0]) and (weights[1, 300].double() - 1 / 64).abs().max() <= 5e-6 / 64
        assert ((loss.double() - want[4]).abs() <= 1e-5 * want[4].abs()).all() and mean.isfinite().all()


@pytest.mark.parametrize("use", [("dw",), ("dl",), ("dw", "dl")], ids="+".join)
@pytest.mark.parametrize("normalize", [False, True])
@pytest.mark.parametrize("E,k", [(6, 2), (8, 8), (64, 8), (64, 9), (130, 4), (300, 1), (1000, 8), (40, 20)])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_route_grad_of_very_large_logits(b, dtype, E, k, normalize, use):
    """Rows are live, whatever finite numbers they hold: no NaN, and no zeros for them."""
    x = extremes(dtype, E)
    G, T = x.shape[:2]
    g = torch.Generator(device="cuda:0")
    g.manual_seed(9)
    chosen, _, counts, _, _ = ref.route(x, k, 0.05, normalize)
    dw = torch.randn(G, T, k, generator=g, device="cuda:0") if "dw" in use else None
    dl = (torch.rand(G, generator=g, device="cuda:0") + 0.5) * T * T if "dl" in use else None
    got = b.prsgd_route_grad(x, chosen.int(), counts.int(), 0.05, normalize=normalize, dweights=dw, dloss=dl)
    want = ref.route_grad(x, chosen, counts, 0.05, normalize, None, dw, dl)
    p = torch.softmax(x.double(), -1)
    # |h| of a token: the balance part's largest, and of the weights' part dw, over the sum of the chosen p where that is divided out
    up = torch.zeros(G, T, 1, dtype=torch.float64, device="cuda:0")
    if dl is not None:
        up += (dl.double() * 0.05 * E / T * counts.amax(1) / (k * T))[:, None, None]
    if dw is not None:
        scale = p.gather(-1, chosen).sum(-1, keepdim=True) if normalize else 1.0
        up += 2 * dw.abs().amax(-1, keepdim=True) / scale
    half = 0.0 if dtype == F32 else torch.finfo(dtype).eps / 2
    tiny = torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
    assert ((got.double() - want).abs() <= 2e-5 * p.amax(-1, keepdim=True) * up + half * want.abs() * 1.01 + tiny).all()
    if "dl" in use and k < E:
        assert (got[0, ::3] != 0).any(-1).all()        # (rows of one value: each has a part of the balance loss's gradient)
