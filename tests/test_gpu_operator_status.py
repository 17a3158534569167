"""prsgd_work_status after each operator that takes a workspace: a workspace needs no particular contents, and what an earlier call or
the memory's last owner left in its status words is not reported for a good call."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def b():
    from paper_1807_06629_b200 import _build
    _build.build_library()
    from paper_1807_06629_b200 import binding
    assert torch.cuda.is_available()
    return binding


def poisoned(t):
    return t.fill_(0xFF)


@pytest.mark.parametrize("k", [2, 9])
@pytest.mark.parametrize("shape", [(1, 1, 16), (2, 0, 16), (0, 5, 16), (3, 40, 16), (2, 3000, 64), (700, 3, 16), (2, 0, 1000)])
def test_after_the_router(b, shape, k):
    x = torch.randn(*shape, device="cuda:0")
    work = poisoned(b.route_workspace(x))
    b.prsgd_route(x, k, 0.1, workspace=work)
    b.prsgd_work_status(work)


@pytest.mark.parametrize("shape", [(2, 10, 100), (2, 200, 300), (0, 4, 4), (2, 0, 4), (2, 4, 0)])
def test_after_the_others(b, shape):
    G = torch.randn(*shape, device="cuda:0")
    work = poisoned(b.orthogonalize_workspace(G))
    b.prsgd_orthogonalize(G, workspace=work)
    b.prsgd_work_status(work)
    poisoned(work)
    b.prsgd_muon_step(G.clone(), torch.zeros_like(G), G, 0.1, workspace=work)
    b.prsgd_work_status(work)


def test_a_workspace_of_nothing_recorded_raises(b):
    """(what the others would report if a call left the words as they were)"""
    with pytest.raises(b.PRSGDError):
        b.prsgd_work_status(torch.full((256,), 0xFF, dtype=torch.uint8, device="cuda:0"))
