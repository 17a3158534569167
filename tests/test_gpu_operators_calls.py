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
