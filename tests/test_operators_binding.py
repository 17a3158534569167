"""The operators' Python functions: what they accept, refuse and size, on tensors that need no GPU."""
import pytest
import torch


@pytest.fixture(scope="module")
def b():
    from paper_1807_06629_b200 import _build
    _build.build_library()
    from paper_1807_06629_b200 import binding
    return binding


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("shape", [(1, 1), (3, 10, 1024), (2, 300, 2500), (4, 500, 1900), (2, 900, 900), (1, 2000, 40)])
def test_a_workspace_serves_results_of_any_type(b, shape, dtype):
    """The call decides its precision by the type of `out`, which the workspace's function does not know."""
    G = torch.empty(shape, dtype=dtype)
    work = b.orthogonalize_workspace(G)
    for out in (torch.float32, torch.bfloat16, torch.float16):
        assert work.numel() >= b.prsgd_orthogonalize_workspace_bytes(*b._size3(G), b._precision_for_result(torch.empty(1, dtype=out)))
    for p in (b.PRECISION_FP32, b.PRECISION_BF16):
        assert b.orthogonalize_workspace(G, p).numel() == b.prsgd_orthogonalize_workspace_bytes(*b._size3(G), p)
