"""Calls of the operators that their documentation allows: workspaces, types and layouts of outputs, masks."""
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


def randn(seed, *shape, dtype=F32):
    g = torch.Generator(device="cuda:0")
    g.manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda:0").to(dtype)


@pytest.mark.parametrize("out_dtype", [F32, BF16, F16])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("shape", [(2, 40, 90), (2, 200, 2500), (1, 300, 270)])
def test_orthogonalize_workspace_for_any_type_of_result(b, shape, dtype, out_dtype):
    G = randn(1, *shape, dtype=dtype)
    work = b.orthogonalize_workspace(G).fill_(0xFF)
    got = b.prsgd_orthogonalize(G, out=torch.empty(shape, dtype=out_dtype, device="cuda:0"), workspace=work)
    b.prsgd_work_status(work)
    assert torch.equal(got, b.prsgd_orthogonalize(G, out=torch.empty(shape, dtype=out_dtype, device="cuda:0")))


def test_a_workspace_is_one_piece_of_memory(b):
    x = randn(2, 2, 40, 16)
    n = b.prsgd_route_workspace_bytes(*x.shape)
    for work in (torch.zeros(1, dtype=torch.uint8, device="cuda:0").expand(n), torch.zeros(2 * n, dtype=torch.uint8, device="cuda:0")[::2], torch.zeros(n, dtype=torch.uint8)):
        with pytest.raises(ValueError, match="workspace must be"):
            b.prsgd_route(x, 2, 0.1, workspace=work)
    words = torch.zeros((n + 3) // 4, dtype=F32, device="cuda:0")       # of any type
    assert all(torch.equal(p, q) for p, q in zip(b.prsgd_route(x, 2, 0.1, workspace=words), b.prsgd_route(x, 2, 0.1)))


def test_a_mask_of_truth_values_is_one_of_bytes(b):
    x, live = randn(3, 3, 50, 24), randn(4, 3, 50) > 0
    got, want = b.prsgd_route(x, 3, 0.1, live=live), b.prsgd_route(x, 3, 0.1, live=live.to(torch.uint8))
    assert all(torch.equal(p, q) for p, q in zip(got, want)) and (got[0][~live] == -1).all()
    kw = dict(dweights=randn(5, 3, 50, 3), dloss=randn(6, 3))
    assert torch.equal(b.prsgd_route_grad(x, got[0], got[2], 0.1, live=live, **kw), b.prsgd_route_grad(x, got[0], got[2], 0.1, live=live.to(torch.uint8), **kw))


def in_turn(t, pad=0):
    """t's values as the matrices of [rows, batch, cols + pad]: a row of each in turn."""
    big = torch.full((t.shape[1], t.shape[0], t.shape[2] + pad), 7.0, dtype=t.dtype, device="cuda:0")
    v = big.transpose(0, 1)[:, :, :t.shape[2]]
    v.copy_(t)
    return v, big


@pytest.mark.parametrize("pad", [0, 3, 8])
@pytest.mark.parametrize("shape", [(3, 40, 96), (3, 70, 33), (2, 200, 300), (4, 300, 136), (1, 40, 40)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_matrices_whose_rows_lie_in_turn(b, dtype, shape, pad):
    """Bounds as in test_gpu_operators.py: 5e-5 (pairs) or 6e-3 (single operands) of the Newton-Schulz part, beside the rounding of the
    type, and of one product and sum for V."""
    G, W, V = randn(10, *shape, dtype=dtype), randn(11, *shape, dtype=dtype), randn(12, *shape)
    tol, half = (5e-5, 0.0) if dtype == F32 else (6e-3, torch.finfo(dtype).eps / 2)
    want = ref.orthogonalize(G)
    near = lambda got: (got.double() - want).norm() <= (tol + half) * want.norm()
    g, g_all = in_turn(G, pad)
    out, out_all = in_turn(torch.zeros_like(G), pad)
    assert near(b.prsgd_orthogonalize(g, out=out)) and (out_all[:, :, shape[2]:] == 7).all()
    w, w_all = in_turn(W, pad)
    v, v_all = in_turn(V, pad)
    want_w, want_v = ref.muon(W, V, G, 0.1, 0.95, True, 0.1, 1.0)
    moved = (want_w - 0.99 * W.double()).norm()
    b.prsgd_muon_step(w, v, g, 0.1, weight_decay=0.1)
    assert (v.double() - want_v).norm() <= 2.0 ** -23 * want_v.norm() and torch.equal(g, G)
    assert (w.double() - want_w).norm() <= tol * moved + max(half, 2.0 ** -23) * want_w.norm()
    assert (w_all[:, :, shape[2]:] == 7).all() and (v_all[:, :, shape[2]:] == 7).all()
    assert near(b.prsgd_orthogonalize(g, out=g)) and (g_all[:, :, shape[2]:] == 7).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_gradients_of_tokens_whose_groups_lie_in_turn(b, dtype):
    x = randn(13, 3, 60, 48, dtype=dtype)
    y, y_all = in_turn(x, 4)
    experts, _, counts, _, _ = got = b.prsgd_route(y, 4, 0.1)
    assert all(torch.equal(p, q) for p, q in zip(got, b.prsgd_route(x, 4, 0.1)))
    kw = dict(dweights=randn(14, 3, 60, 4), dloss=randn(15, 3))
    want = b.prsgd_route_grad(x, experts, counts, 0.1, **kw)
    assert torch.equal(b.prsgd_route_grad(y, experts, counts, 0.1, out=y, **kw), want) and (y_all[:, :, 48:] == 7).all()
