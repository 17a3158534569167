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


def not_one_piece():
    return [torch.zeros(1, dtype=torch.uint8).expand(1 << 24), torch.zeros(1 << 12, 1 << 12, dtype=torch.uint8).t()[::2]]


def test_a_workspace_is_one_piece_of_memory(b):
    """A view whose elements share memory, or lie apart, is larger by its count than what it may be written through."""
    G = torch.zeros(2, 10, 100)
    for work in not_one_piece():
        with pytest.raises(ValueError, match="workspace must be"):
            b.prsgd_orthogonalize(G, out=G, workspace=work)
        with pytest.raises(ValueError, match="workspace must be"):
            b.prsgd_muon_step(G, G.clone(), G.clone(), 0.1, workspace=work)
        with pytest.raises(ValueError, match="workspace must be"):
            b._scratch(work, -1)
    words = torch.zeros(100, dtype=torch.float32)
    assert b._scratch(words, -1) == (words.data_ptr(), 400)


def test_a_mask_is_bytes_or_truth_values(b):
    for dtype in (torch.uint8, torch.bool):
        live = torch.zeros(3, 4, dtype=dtype)
        assert b._mask(live, 12, -1) == live.data_ptr()
    assert b._mask(None, 12, -1) is None
    for bad in (torch.zeros(3, 4, dtype=torch.int32), torch.zeros(3, 5, dtype=torch.bool), torch.zeros(4, 3, dtype=torch.bool).t()):
        with pytest.raises(ValueError, match="live"):
            b._mask(bad, 12, -1)


def test_coefficients_are_three(b):
    assert b._coefs(None) is None and b._coefs(list(b.MUON_COEFS)) is None and list(b._coefs((1.5, -0.5, 0.0))) == [1.5, -0.5, 0.0]
    for bad in ((), (1.5,), (1.5, -0.5), (1.5, -0.5, 0.0, 0.0)):
        with pytest.raises(ValueError, match="coefs"):
            b._coefs(bad)
